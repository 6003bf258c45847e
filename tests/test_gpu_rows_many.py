"""Tokens to rows and back as the calls go about many tokens: with one or two choices several vectors a thread, several tokens a CTA, rows over more CTAs than one, parts of
rows that end in the middle, rows of 8 bits that end on 8 bytes. Sizes are those from which these forms are taken on 148 SMs; bounds are test_gpu_rows'."""
import pytest
import torch

import paper_2605_26845_b200 as ms
from test_gpu_rows import bits, check_back, random, slots

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = [(1, 2501, 1, 264), (1, 9001, 1, 512), (1, 1300, 1, 2056), (3, 901, 2, 1032), (1, 2501, 2, 264), (1, 401, 2, 7168), (1, 5003, 3, 136), (2, 1201, 4, 264), (1, 601, 4, 4104),
         (2, 1501, 5, 520), (1, 1201, 7, 2056), (1, 400, 8, 7168), (1, 999, 9, 4104), (1, 2400, 17, 72)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,T,k,D", SIZES)
def test_back_and_gradients(G, T, k, D, dtype):
    check_back(G, T, k, D, TYPES[dtype], True, True, seed=T + D)
    check_back(G, T, k, D, TYPES[dtype], False, False, seed=T + D)


@pytest.mark.parametrize("dtype", [*TYPES.values(), torch.float8_e4m3fn, torch.uint8])
@pytest.mark.parametrize("G,T,k,D", SIZES)
def test_to_rows(G, T, k, D, dtype):
    x, slot, scale = random(dtype, G, T, D, seed=D), slots(G, T, k, T), random(torch.float32, G, T, 5, seed=k)
    token = torch.arange(T * k, device="cuda") // k
    rows, moved = torch.full((G, T * k, D), 7, dtype=torch.uint8, device="cuda").to(dtype), torch.full((G, T * k, 5), 7.0, device="cuda")
    want, want_scale = bits(rows).clone(), moved.clone()
    for b in range(G):
        sent = slot[b] >= 0
        want[b, slot[b][sent].long()] = bits(x)[b, token[sent]]
        want_scale[b, slot[b][sent].long()] = scale[b, token[sent]]
    ms.tokens_to_rows(x, slot, scale=scale, out=rows, out_scale=moved)
    assert torch.equal(bits(rows), want) and torch.equal(moved, want_scale)
    rows.view(torch.uint8).fill_(9)
    ms.tokens_to_rows(x, slot, out=rows)
    left = torch.ones((G, T * k), dtype=torch.bool, device="cuda")
    for b in range(G):
        left[b, slot[b][slot[b] >= 0].long()] = False
    assert torch.equal(bits(rows)[~left], want[~left]) and (bits(rows)[left] == 9).all()


def test_a_layer_of_one_choice_in_a_graph():
    """Many tokens, forward and backward, captured twice: the graphs share nothing."""
    T, D = 3001, 520
    x, dy, slot = random(torch.bfloat16, T, D, seed=1), random(torch.bfloat16, T, D, seed=2), slots(1, T, 1, 3)[0]
    w = torch.rand(T, device="cuda")

    def run():
        rows = ms.tokens_to_rows(x, slot, out=torch.zeros((T, D), dtype=torch.bfloat16, device="cuda"))
        return rows, ms.rows_to_tokens(rows, slot, 1, weights=w, add=x), *ms.rows_to_tokens_backward(dy, rows, slot, w, out={"drows": torch.zeros_like(rows)}).values()

    want, graphs = run(), []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((run(), graph))
    for stream, (_, graph) in zip((torch.cuda.Stream(), torch.cuda.Stream()), graphs):
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            graph.replay()
            graph.replay()
        torch.cuda.current_stream().wait_stream(stream)
    for got, _ in graphs:
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
