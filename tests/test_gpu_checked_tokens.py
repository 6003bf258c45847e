"""The kernels on tokens in the range-checked build: what they take from data for an index (candidates' places, chosen experts, slots) stays in range, and the results are
those of the regular build, bit for bit."""
import pytest
import torch

import paper_2605_26845_b200 as ms
from paper_2605_26845_b200 import build as cuda_build

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture
def both():
    """Runs a call with the regular and with the checked library, and compares."""
    def run(call):
        want = call()
        ms.use_library(cuda_build.build(checked=True))
        try:
            assert ms.debug_index_faults() == 0
            got = call()
            assert ms.debug_index_faults() == 0
        finally:
            ms.use_library(None)
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    return run


def logits(T, E, kind, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    l = torch.randn((T, E), generator=g, device="cuda")
    if kind == "ties":
        return torch.randint(-1, 2, (T, E), generator=g, device="cuda").float()
    if kind == "equal":                                     # more than 32 candidates
        return torch.full((T, E), 0.25, device="cuda")
    if kind == "near":                                      # scores that 32 bits do not tell apart
        return 1 + torch.randint(0, 4, (T, E), generator=g, device="cuda").float() * 2.0 ** -23
    if kind == "off":
        l[torch.rand((T, E), generator=g, device="cuda") < 0.9] = -INF
        l[0], l[-1, 0], l[T // 2, -1] = -INF, NAN, INF
    return l


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "near", "off"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (9, 7, 7), (33, 31, 5), (17, 32, 32), (50, 60, 6), (19, 128, 8), (600, 256, 8), (11, 257, 9), (5, 1000, 32), (7, 1024, 3)])
def test_choices_stay_in_range(both, T, E, k, kind):
    l = logits(T, E, kind, E + k)
    dw = torch.randn(T * k, device="cuda", generator=torch.Generator("cuda").manual_seed(1))

    def call():
        res = []
        for score in ("softmax", "sigmoid"):
            for normalise in (False, True):
                for bias in (None, torch.zeros(E, device="cuda"), torch.linspace(0.3, -0.3, E, device="cuda")):
                    got = ms.route_choose(l, k, score=score, bias=bias, normalise=normalise)
                    res += [got["experts"], got["weights"], ms.route_choose_backward(dw, l, got["experts"], score=score, normalise=normalise)]
        wrong = torch.randint(-5, E + 5, (T * k,), device="cuda", dtype=torch.int32, generator=torch.Generator("cuda").manual_seed(2)).sort().values
        return res + [ms.route_choose_backward(dw[:T], l, wrong[:T].contiguous())]      # (entries outside 0 .. E - 1 were not chosen)

    both(call)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,T,k,D", [(1, 1, 1, 8), (2, 3, 2, 16), (3, 16, 5, 264), (1, 300, 8, 2048), (2, 700, 3, 136), (1, 2501, 2, 1032)])
def test_slots_stay_in_range(both, G, T, k, D, dtype):
    g = torch.Generator("cuda").manual_seed(T)
    S = T * k
    slot = torch.rand((G, S), generator=g, device="cuda").argsort(-1).int()
    lost = torch.rand((G, S), generator=g, device="cuda") < 0.2
    slot[lost] = torch.randint(0, 4, (G, S), generator=g, device="cuda", dtype=torch.int32)[lost] * (1 << 29) + S      # (beyond the source's rows)
    x, back = (torch.randn((G, n, D), generator=g, device="cuda").to(dtype) for n in (T, S))
    w, scale = torch.rand((G, S), generator=g, device="cuda"), torch.rand((G, T, 2), generator=g, device="cuda")

    def call():
        rows, moved = ms.tokens_to_rows(x, slot, scale=scale, out=torch.zeros_like(back), out_scale=torch.zeros((G, S, 2), device="cuda"))
        grads = ms.rows_to_tokens_backward(x, back, slot, w, out={"drows": torch.zeros_like(back)})
        eight = ms.tokens_to_rows(x.to(torch.float8_e4m3fn), slot, out=torch.zeros((G, S, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn))
        return rows, moved, ms.rows_to_tokens(back, slot, k, weights=w, add=x), grads["drows"], grads["dweights"], eight.view(torch.uint8)

    both(call)
