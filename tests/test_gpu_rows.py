"""Tokens to rows by expert and back. What is moved has to be equal; sums against 64 bits: a sum of n products in 32 bits is off by at most n + 1 half steps (2^-24) of
the sum of magnitudes, then half a step of the type."""
import pytest
import torch

import paper_2605_26845_b200 as ms
from test_gpu_expert import Rounded

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = 2.0 ** -24


def slots(G, T, k, seed, dropped=0.1):
    """Distinct slots of every source, some choices without one."""
    g = torch.Generator("cuda").manual_seed(seed)
    slot = torch.rand((G, T * k), generator=g, device="cuda").argsort(-1).int()
    return torch.where(torch.rand((G, T * k), generator=g, device="cuda") < dropped, -1, slot).contiguous()


def random(dtype, *shape, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    if dtype == torch.uint8:
        return torch.randint(0, 256, shape, generator=g, device="cuda", dtype=dtype)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def bits(t):
    return t.view(torch.uint8)


def near(got, want, err, what):
    off = (got.double() - want).abs() - err
    assert torch.isfinite(got).all(), what
    assert (off <= 0).all(), (what, off.max().item())


SIZES = [(1, 1, 1, 8), (1, 1, 8, 7168), (2, 3, 2, 16), (1, 37, 3, 1000), (3, 16, 5, 264), (1, 5, 32, 72), (4, 61, 6, 1032), (1, 300, 8, 2048), (2, 7, 9, 4104), (1, 2, 4, 65536)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.uint8])
@pytest.mark.parametrize("G,T,k,D", SIZES)
def test_tokens_to_rows(G, T, k, D, dtype):
    x, slot = random(dtype, G, T, D, seed=D), slots(G, T, k, T)
    rows = torch.full((G, T * k, D), 7, dtype=torch.uint8, device="cuda").to(dtype)
    want = bits(rows).clone()
    token = torch.arange(T * k, device="cuda") // k
    for b in range(G):
        sent = slot[b] >= 0
        want[b, slot[b][sent].long()] = bits(x)[b, token[sent]]
    assert ms.tokens_to_rows(x, slot, out=rows) is rows
    assert torch.equal(bits(rows), want)
    if G == 1:                                              # one source without a dimension of its own
        alone = torch.full_like(rows[0].float(), 7).to(dtype)
        assert torch.equal(bits(ms.tokens_to_rows(x[0], slot[0], out=alone)), want[0])
    for P in (1, 3, -(-D // 32)):
        scale = random(torch.float32, G, T, P, seed=P)
        if P > D:
            continue
        into = torch.full((G, T * k, P), 7.0, device="cuda")
        rows.fill_(7)
        got, moved = ms.tokens_to_rows(x, slot, scale=scale, out=rows, out_scale=into)
        assert moved is into and torch.equal(bits(got), want)
        for b in range(G):
            sent = slot[b] >= 0
            left = torch.ones(T * k, dtype=torch.bool, device="cuda")
            left[slot[b][sent].long()] = False
            assert torch.equal(moved[b, slot[b][sent].long()], scale[b, token[sent]]) and (moved[b, left] == 7).all()


def check_back(G, T, k, D, dtype, weighted, added, seed=0, dropped=0.1):
    rows, slot = random(dtype, G, T * k, D, seed=seed + 1), slots(G, T, k, seed, dropped)
    w = torch.rand((G, T * k), generator=torch.Generator("cuda").manual_seed(seed), device="cuda") - 0.3 if weighted else None
    add, dy = random(dtype, G, T, D, seed=seed + 2) if added else None, random(dtype, G, T, D, seed=seed + 3)
    rnd = Rounded(dtype)
    sent = slot >= 0
    picked = torch.stack([rows[b][slot[b].clamp_min(0).long()] for b in range(G)]).double() * sent[..., None]
    terms = (picked * (w.double()[..., None] if weighted else 1.0)).view(G, T, k, D)
    want = terms.sum(2) + (add.double() if added else 0)
    size = terms.abs().sum(2) + (add.double().abs() if added else 0)
    y = ms.rows_to_tokens(rows, slot, k, weights=w, add=add)
    near(y, want, rnd(want, (k + 1) * U * size), "y")
    if added:
        own = add.clone()
        assert ms.rows_to_tokens(rows, slot, k, weights=w, add=own, out=own) is own and torch.equal(own, y)
    if not weighted:
        return
    for name in ("new", "rows"):
        source = rows.clone()
        into = source if name == "rows" else torch.full_like(rows, 7)
        before = into.clone()
        got = ms.rows_to_tokens_backward(dy, source, slot, w, out={"drows": into})
        assert got["drows"] is into
        for b in range(G):
            at, token = slot[b][sent[b]].long(), (torch.arange(T * k, device="cuda") // k)[sent[b]]
            exact = dy[b].double()[token] * w[b].double()[sent[b]][:, None]
            near(into[b][at], exact, rnd(exact, U * exact.abs()), "drows")
            left = torch.ones(T * k, dtype=torch.bool, device="cuda")
            left[at] = False
            assert torch.equal(into[b][left], before[b][left])
        each = picked.view(G, T, k, D) * dy.double()[:, :, None]
        near(got["dweights"], each.sum(-1).view(G, T * k), (D + 1) * U * each.abs().sum(-1).view(G, T * k), "dweights")
        assert (got["dweights"][~sent] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,T,k,D", SIZES)
def test_rows_to_tokens_and_gradients(G, T, k, D, dtype):
    for weighted in (False, True):
        for added in (False, True):
            check_back(G, T, k, D, TYPES[dtype], weighted, added, seed=D + T)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [8, 136, 256, 512, 1024, 1160, 2056, 3080, 4096, 7168, 8200, 16384, 32776])
def test_widths(D, dtype):
    for k in (1, 2, 8):
        check_back(1, 9, k, D, TYPES[dtype], True, True, seed=D)


def test_tokens_without_any_row():
    for dtype in TYPES.values():
        check_back(2, 40, 3, 136, dtype, True, True, seed=5, dropped=0.8)
        rows, slot = random(dtype, 12, 64), torch.full((12,), -1, dtype=torch.int32, device="cuda")
        w, add = torch.ones(12, device="cuda"), random(dtype, 4, 64, seed=3)
        assert (ms.rows_to_tokens(rows, slot, 3, weights=w) == 0).all()
        assert torch.equal(ms.rows_to_tokens(rows, slot, 3, weights=w, add=add), add)
        got = ms.rows_to_tokens_backward(add, rows, slot, w, out={"drows": rows.clone()})
        assert (got["dweights"] == 0).all() and torch.equal(got["drows"], rows)


def test_what_was_not_sent_counts_for_nothing():
    """Neither the weight of such a choice nor what lies in unused rows is looked at, and a slot beyond the source's rows is one of them."""
    slot = torch.tensor([2, -1, 6, 0, -2147483648, 2147483647], dtype=torch.int32, device="cuda")
    rows, w = random(torch.float32, 6, 64), torch.tensor([0.5, float("nan"), float("inf"), 2.0, float("nan"), 1.0], device="cuda")
    rows[1], rows[3:] = float("nan"), float("inf")
    y = ms.rows_to_tokens(rows, slot, 2, weights=w)
    assert torch.equal(y, torch.stack([0.5 * rows[2], 2 * rows[0], torch.zeros_like(rows[0])])[[0, 1, 2]].index_copy(0, torch.tensor([1, 2], device="cuda"), torch.stack([2 * rows[0], 0 * rows[0]])))
    dy = random(torch.float32, 3, 64, seed=1)
    got = ms.rows_to_tokens_backward(dy, rows, slot, w, out={"drows": torch.full_like(rows, 7)})
    assert (got["drows"][[1, 3, 4, 5]] == 7).all() and torch.equal(got["drows"][2], 0.5 * dy[0]) and torch.equal(got["drows"][0], 2 * dy[1])
    assert (got["dweights"][[1, 2, 4, 5]] == 0).all()
    out = ms.tokens_to_rows(dy, slot, out=torch.full_like(rows, 7))
    assert (out[[1, 3, 4, 5]] == 7).all() and torch.equal(out[2], dy[0]) and torch.equal(out[0], dy[1])


def test_infinities_and_nan_of_rows_that_were_sent_go_on():
    slot = torch.arange(4, dtype=torch.int32, device="cuda")
    for dtype in TYPES.values():
        rows = random(dtype, 4, 64)
        rows[0, 3], rows[2, 5] = float("inf"), float("nan")
        y = ms.rows_to_tokens(rows, slot, 2, weights=torch.ones(4, device="cuda"))
        assert y[0, 3] == float("inf") and torch.isnan(y[1, 5]) and torch.isfinite(y[0, :3]).all()


def test_the_gradient_of_sending_is_the_sum_of_what_comes_back():
    x, slot = random(torch.float32, 2, 20, 72), slots(2, 20, 4, 3)
    drows = random(torch.float32, 2, 80, 72, seed=2)
    rows = ms.tokens_to_rows(x, slot, out=torch.zeros_like(drows))
    dx = ms.rows_to_tokens(drows, slot, 4)
    named = torch.zeros((2, 80), device="cuda")
    for b in range(2):
        named[b, slot[b][slot[b] >= 0].long()] = 1
    left, right = (rows.double() * drows.double() * named[..., None]).sum(), (x.double() * dx.double()).sum()
    assert abs(left - right) <= 5 * U * (rows.double() * drows.double()).abs().sum()      # <A x, d> = <x, A' d>, sums of four


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D,group", [(1, 8, 32), (3, 72, 64), (40, 1000, 128), (300, 1032, 32), (77, 7168, 128), (5, 65536, 64)])
def test_rows_widen(R, D, group, dtype):
    every = torch.arange(256, device="cuda", dtype=torch.uint8)
    every = every[(every & 127) != 127]                     # (those are NaN)
    g = torch.Generator("cuda").manual_seed(R)
    q = every[torch.randint(0, 254, (R, D), generator=g, device="cuda")].view(torch.float8_e4m3fn)
    scale = torch.rand((R, -(-D // group)), generator=g, device="cuda") * 2 + 2.0 ** -126
    got = ms.rows_widen(q, scale, group, TYPES[dtype])
    want = q.double() * scale.double().repeat_interleave(group, 1)[:, :D]
    near(got, want, Rounded(TYPES[dtype])(want, U * want.abs()), "widen")
    bad = q.view(torch.uint8).clone()
    bad[0, 3] = 127
    assert torch.isnan(ms.rows_widen(bad.view(torch.float8_e4m3fn), scale, group, TYPES[dtype])[0, 3])
    deep = ms.rows_widen(q.view(1, R, D), scale.view(1, R, -1), group, TYPES[dtype])
    assert torch.equal(deep[0], got)


def test_buffers_beyond_32_bits():
    """4.3 thousand million values of rows: places are counted in 64 bits."""
    T, k, D = 1 << 17, 8, 4096
    x = random(torch.uint8, T, D)
    slot = slots(1, T, k, 1, dropped=0.001)[0]
    scale = random(torch.float32, T, 32)
    rows, moved = ms.tokens_to_rows(x, slot, scale=scale)
    for choice in torch.randint(0, T * k, (200,), generator=torch.Generator().manual_seed(1)).tolist() + slot.topk(5).indices.tolist():
        if slot[choice] >= 0:
            assert torch.equal(rows[slot[choice]], x[choice // k]) and torch.equal(moved[slot[choice]], scale[choice // k])
    del x, moved
    rows = rows.view(torch.float8_e4m3fn)
    wide = ms.rows_widen(rows, torch.ones((T * k, 32), device="cuda"), 128)
    for row in (0, 1 << 19, T * k - 1):
        assert torch.equal(wide[row].float().nan_to_num(9), rows[row].float().nan_to_num(9))
    del rows
    w, dy = torch.rand(T * k, device="cuda"), random(torch.bfloat16, T, D, seed=5)
    wide.nan_to_num_(0)                                     # (bytes at random)
    last = int(slot.argmax()) // k
    first = wide[slot[last * k:(last + 1) * k].clamp_min(0).long()].double() * (slot[last * k:(last + 1) * k] >= 0)[:, None]
    y = ms.rows_to_tokens(wide, slot, k, weights=w)
    want = (first * w[last * k:(last + 1) * k].double()[:, None])
    near(y[last], want.sum(0), Rounded(torch.bfloat16)(want.sum(0), 9 * U * want.abs().sum(0)), "y")
    got = ms.rows_to_tokens_backward(dy, wide, slot, w, out={"drows": wide})
    dots = first * dy[last].double()
    near(got["dweights"][last * k:(last + 1) * k], dots.sum(-1), (D + 1) * U * dots.abs().sum(-1), "dweights")
    for choice in (int(slot.argmax()), int((slot == 1 << 19).nonzero()[0]) if (slot == 1 << 19).any() else 0):
        exact = dy[choice // k].double() * w[choice].double()
        near(wide[slot[choice]], exact, Rounded(torch.bfloat16)(exact, U * exact.abs()), "drows")


def test_captured_calls_and_another_stream():
    x, slot, w = random(torch.bfloat16, 61, 1032), slots(1, 61, 6, 2)[0], torch.rand(366, device="cuda")
    rows = torch.zeros((366, 1032), dtype=torch.bfloat16, device="cuda")
    dr = torch.zeros_like(rows)

    def run():
        ms.tokens_to_rows(x, slot, out=rows)
        y = ms.rows_to_tokens(rows, slot, 6, weights=w, add=x)
        return y, ms.rows_to_tokens_backward(x, rows, slot, w, out={"drows": dr})["dweights"]

    want = [t.clone() for t in (*run(), rows, dr)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    rows.zero_()
    dr.zero_()
    for _ in range(2):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((*got, rows, dr), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, rows, dr), want))
