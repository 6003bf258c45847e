"""Demand from the router's choices, and the places of a schedule's tokens, against plain loops over Python integers."""
import numpy as np
import pytest
import torch

import paper_2605_26845_b200 as ms
from paper_2605_26845_b200.workload import bvn_capacity, random_matrices

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def plain_route(experts, E):
    B, N, S = experts.shape
    P = E // N
    counts, slot = np.zeros((B, N, E), np.int32), np.full((B, N, S), -1, np.int32)
    for b in range(B):
        for i in range(N):
            e = experts[b, i]
            sent = np.flatnonzero((e >= 0) & (e < E))
            counts[b, i] = np.bincount(e[sent], minlength=E)
            slot[b, i, sent[np.argsort(e[sent], kind="stable")]] = np.arange(sent.size)
    return counts.reshape(B, N, N, P).sum(-1, dtype=np.int32), counts, slot


def plain_slots(D, perm, dur, count, counts=None):
    B, K, N = perm.shape
    P = counts.shape[2] // N if counts is not None else 0
    start, length, row = (np.zeros((B, K, N), np.int32) for _ in range(3))
    rows, offsets = np.zeros((B, N), np.int32), np.zeros((B, N, K * P + 1), np.int32)
    for b in range(B):
        left, have = D[b].astype(np.int64), np.zeros(N, np.int64)
        for k in range(K):
            if k >= count[b]:
                offsets[b, :, k * P:] = have[:, None]
                continue
            for i in range(N):
                j = int(perm[b, k, i])
                n = min(left[i, j], int(dur[b, k]))
                start[b, k, i], length[b, k, i], row[b, k, i] = D[b, i, j] - left[i, j], n, have[j]
                if P:
                    ahead = np.concatenate([[0], np.cumsum(counts[b, i, j * P:(j + 1) * P], dtype=np.int64)[:-1]])
                    offsets[b, j, k * P:(k + 1) * P] = have[j] + np.clip(ahead - start[b, k, i], 0, n)
                left[i, j] -= n
                have[j] += n
        rows[b] = have
        offsets[b, :, -1] = have
    return dict(start=start, length=length, row=row, rows=rows, **({"offsets": offsets} if P else {}))


def split(D, P, seed):
    """Choices by expert with the sums D."""
    rng = np.random.default_rng(seed)
    share = rng.random(D.shape + (P,)) * (rng.random(D.shape + (P,)) < 0.7)
    cut = np.floor(D[..., None] * np.cumsum(share, -1) / np.maximum(share.sum(-1, keepdims=True), 1e-9)).astype(np.int64)
    cut[..., -1] = D
    return np.diff(cut, axis=-1, prepend=0).astype(np.int32).reshape(D.shape[0], D.shape[1], -1)


def same(got, want):
    assert (got["status"] == 0).all()
    for k, v in want.items():
        assert (got[k].cpu().numpy() == v).all(), k


@pytest.mark.parametrize("B,N,S,P", [(1, 1, 1, 1), (2, 1, 0, 3), (3, 2, 31, 1), (1, 8, 8192, 1), (2, 5, 1025, 3), (2, 16, 4099, 4), (1, 64, 777, 16),
                                     (1, 256, 129, 4), (1, 3, 131072, 341), (40, 7, 33, 2), (1, 2, 300_001, 5)])
def test_route_demand(B, N, S, P):
    rng = np.random.default_rng(100 * N + S)
    E = N * P
    e = np.minimum(rng.zipf(1.3, size=(B, N, S)) - 1, E - 1)
    e = np.where(rng.random(e.shape) < 0.1, -1, rng.permutation(E)[e]).astype(np.int32)
    got = ms.route_demand(dev(e), E)
    same(got, dict(zip(("demand", "counts", "slot"), plain_route(e, E))))
    again = ms.route_demand(dev(e), E, out={k: torch.full_like(v, 77) for k, v in got.items()})
    assert all((got[k] == again[k]).all() for k in got)


def test_one_expert_takes_everything_and_nothing_is_sent():
    for fill in (0, 11, -1):
        e = np.full((2, 3, 5000), fill, np.int32)
        same(ms.route_demand(dev(e), 12), dict(zip(("demand", "counts", "slot"), plain_route(e, 12))))


def test_choices_out_of_range_are_not_sent_and_their_source_is_marked():
    e = np.random.default_rng(1).integers(0, 24, size=(2, 6, 3001)).astype(np.int32)
    e[0, 3, 7], e[0, 3, 2999], e[1, 5, 0], e[1, 0, 9] = 24, -2, 2 ** 31 - 1, -2 ** 31
    got = ms.route_demand(dev(e), 24)
    status = np.zeros((2, 6), np.int32)
    status[0, 3] = status[1, 5] = status[1, 0] = ms.ST_BAD_INPUT
    assert (got["status"].cpu().numpy() == status).all()
    for k, v in zip(("demand", "counts", "slot"), plain_route(e, 24)):
        assert (got[k].cpu().numpy() == v).all(), k


@pytest.mark.parametrize("N", [1, 2, 3, 7, 8, 16, 31, 32, 33, 64, 65, 100, 128, 129, 130, 200, 256])
@pytest.mark.parametrize("kind", ["greedy", "birkhoff"])
def test_schedule_slots(N, kind):
    D = random_matrices(3, N, seed=500 + N, kind="uniform", high=900, zero_frac=0.3)
    d = dev(D)
    s = ms.mw_decompose(d, min(2 * N, 90)) if kind == "greedy" else ms.bvn_decompose(d, min(bvn_capacity(N), 131))
    perm, dur, count = (t.cpu().numpy() for t in (s.perm, s.dur, s.count))
    if N > 1:
        count[1] //= 2                                    # some tokens are left behind
        s.count[1] = int(count[1])
    for P in (1, 3):
        if N * P <= ms.MAX_EXPERTS:
            counts = split(D, P, N)
            same(ms.schedule_slots(d, s.perm, s.dur, s.count, dev(counts)), plain_slots(D, perm, dur, count, counts))
    got = ms.schedule_slots(d, s.perm, s.dur, s.count)
    same(got, plain_slots(D, perm, dur, count))
    score = ms.schedule_eval(d, s.perm, s.dur, s.count)   # the same replay
    left = d.sum((1, 2), dtype=torch.int64) - got["length"].sum((1, 2), dtype=torch.int64)
    assert (score["unserved_tokens"] == left).all()


@pytest.mark.parametrize("P", [3, 4])
@pytest.mark.parametrize("B,N,K", [(1, 4, 700), (2, 8, 333), (1, 64, 500), (3, 100, 260), (1, 128, 1000), (2, 16, 64), (1, 17, 33), (40, 12, 129), (200, 6, 40)])
def test_repeated_pairs_and_long_schedules(B, N, K, P):
    """Random permutations and durations: the pairs come back in any distance, also within 32 matchings, and after they are empty."""
    rng = np.random.default_rng(K)
    D = rng.integers(0, 200, size=(B, N, N)).astype(np.int32)
    D[0, 0] = 2 ** 31 // N - 5                            # rows up to nearly 2^31 - 1
    perm = np.stack([np.stack([rng.permutation(N) for _ in range(K)]) for _ in range(B)]).astype(np.uint8)
    perm[0, 3:9] = perm[0, 2]
    dur = rng.integers(0, 60, size=(B, K)).astype(np.int32)
    dur[0, 5:8] = 2 ** 31 - 1
    count = rng.integers(K - K // 4, K + 1, size=B).astype(np.int32)
    count[-1] = K
    counts = split(D, P, K)
    same(ms.schedule_slots(dev(D), dev(perm), dev(dur), dev(count), dev(counts)), plain_slots(D, perm, dur, count, counts))


def test_empty_schedules():
    d, perm = torch.ones((4, 9, 9), dtype=torch.int32, device="cuda"), torch.zeros((4, 5, 9), dtype=torch.uint8, device="cuda")
    counts = torch.ones((4, 9, 9), dtype=torch.int32, device="cuda")
    z = torch.zeros(4, dtype=torch.int32, device="cuda")
    got = ms.schedule_slots(d, perm, torch.ones((4, 5), dtype=torch.int32, device="cuda"), z, counts)
    assert all((v == 0).all() for v in got.values())


@pytest.mark.parametrize("K", [70, 300])
@pytest.mark.parametrize("N", [6, 40, 128, 160])
def test_rejected_schedules_are_all_zero(N, K):
    B, P = 8, 2
    rng = np.random.default_rng(N)
    D = rng.integers(1, 50, size=(B, N, N)).astype(np.int32)
    perm = np.stack([np.stack([rng.permutation(N) for _ in range(K)]) for _ in range(B)]).astype(np.uint8)
    dur, count = rng.integers(1, 60, size=(B, K)).astype(np.int32), np.full(B, K, np.int32)
    counts = split(D, P, N)
    D[1, N - 1, 2] = -1
    perm[2, 68, 0] = perm[2, 68, 1]
    count[3] = K + 1
    dur[4, K - 1] = -5
    i, j = 3, int(perm[5, 0, 3])
    counts[5, i, j * P] += 1                              # sums to more than the pair has
    count[6] = -1
    perm[7, 3, 2] = N if N < 256 else perm[7, 3, 1]
    got = ms.schedule_slots(dev(D), dev(perm), dev(dur), dev(count), dev(counts))
    assert got["status"].tolist() == [0] + [ms.ST_BAD_INPUT] * 7
    for k, v in plain_slots(D[:1], perm[:1], dur[:1], count[:1], counts[:1]).items():
        assert (got[k][:1].cpu().numpy() == v).all() and (got[k][1:] == 0).all(), k


def test_more_rows_than_an_int32_counts_are_rejected():
    N = 4
    D = np.full((2, N, N), 2 ** 30, np.int32)
    D[1] -= 2 ** 29 + 1
    perm = np.stack([(np.arange(N) + k) % N for k in range(N)]).astype(np.uint8)[None].repeat(2, 0)
    dur, count = np.full((2, N), 2 ** 31 - 1, np.int32), np.full(2, N, np.int32)
    got = ms.schedule_slots(dev(D), dev(perm), dev(dur), dev(count))
    assert got["status"].tolist() == [ms.ST_BAD_INPUT, 0]
    assert (got["rows"][0] == 0).all() and (got["rows"][1] == 4 * (2 ** 29 - 1)).all()


def test_the_checked_build_sees_no_index_out_of_range():
    from paper_2605_26845_b200 import build as cuda_build
    ms.use_library(cuda_build.build(checked=True))
    try:
        before = ms.debug_index_faults()
        for N, K in ((5, 100), (64, 200), (150, 70)):
            rng = np.random.default_rng(N)
            D = rng.integers(0, 50, size=(2, N, N)).astype(np.int32)
            perm = np.stack([np.stack([rng.permutation(N) for _ in range(K)]) for _ in range(2)]).astype(np.uint8)
            dur, count = rng.integers(0, 9, size=(2, K)).astype(np.int32), np.full(2, K, np.int32)
            same(ms.schedule_slots(dev(D), dev(perm), dev(dur), dev(count)), plain_slots(D, perm, dur, count))
            e = rng.integers(-1, 3 * N, size=(2, N, 999)).astype(np.int32)
            same(ms.route_demand(dev(e), 3 * N), dict(zip(("demand", "counts", "slot"), plain_route(e, 3 * N))))
        assert ms.debug_index_faults() == before == 0
    finally:
        ms.use_library(None)


def test_on_another_stream_and_replayed_from_a_graph():
    rng = np.random.default_rng(3)
    e = dev(rng.integers(-1, 32, size=(2, 8, 2000)).astype(np.int32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = ms.route_demand(e, 32)
        s = ms.mw_decompose(r["demand"], 8)
        got = ms.schedule_slots(r["demand"], s.perm, s.dur, s.count, r["counts"])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r2 = ms.route_demand(e, 32)
        s2 = ms.mw_decompose(r2["demand"], 8)
        got2 = ms.schedule_slots(r2["demand"], s2.perm, s2.dur, s2.count, r2["counts"])
    for seed in (4, 5):
        e.copy_(dev(np.random.default_rng(seed).integers(-1, 32, size=(2, 8, 2000)).astype(np.int32)))
        graph.replay()
        demand, counts, slot = plain_route(e.cpu().numpy(), 32)
        same(r2, dict(demand=demand, counts=counts, slot=slot))
        same(got2, plain_slots(demand, *(t.cpu().numpy() for t in (s2.perm, s2.dur, s2.count)), counts))
    assert (got["rows"].sum(1) == r["demand"].sum((1, 2))).all()


@pytest.mark.parametrize("N,P", [(5, 1), (5, 2), (64, 4), (60, 7), (16, 8), (33, 9), (7, 12), (85, 12), (128, 8), (200, 4), (200, 5), (3, 341), (1, 1024)])
@pytest.mark.parametrize("B,K", [(2, 40), (1, 300)])
def test_any_number_of_experts_on_a_rank(N, P, B, K):
    rng = np.random.default_rng(N * P)
    D = rng.integers(0, 300, size=(B, N, N)).astype(np.int32)
    perm = np.stack([np.stack([rng.permutation(N) for _ in range(K)]) for _ in range(B)]).astype(np.uint8)
    dur, count = rng.integers(0, 90, size=(B, K)).astype(np.int32), np.full(B, K - 3, np.int32)
    counts = split(D, P, K)
    want = plain_slots(D, perm, dur, count, counts)
    same(ms.schedule_slots(dev(D), dev(perm), dev(dur), dev(count), dev(counts)), want)
    # tensors that do not begin at 16 bytes
    def shifted(a):
        flat = torch.zeros(a.size + 1, dtype=dev(a).dtype, device="cuda")
        flat[1:] = dev(a).reshape(-1)
        return flat[1:].view(a.shape)
    same(ms.schedule_slots(*(shifted(a) for a in (D, perm, dur, count, counts))), want)


def test_a_batch_of_no_matrices():
    z = torch.zeros((0, 4, 4), dtype=torch.int32, device="cuda")
    assert ms.route_demand(torch.zeros((0, 4, 9), dtype=torch.int32, device="cuda"), 8)["demand"].shape == (0, 4, 4)
    got = ms.schedule_slots(z, torch.zeros((0, 3, 4), dtype=torch.uint8, device="cuda"), torch.zeros((0, 3), dtype=torch.int32, device="cuda"),
                            torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros((0, 4, 8), dtype=torch.int32, device="cuda"))
    assert got["offsets"].shape == (0, 4, 7)


def test_numbers_of_experts_that_do_not_fit():
    e = torch.zeros((1, 4, 9), dtype=torch.int32, device="cuda")
    for experts in (-4, 0, 2, 6, 1028):
        with pytest.raises(ms.MoeschedError):
            ms.route_demand(e, experts)


@pytest.mark.parametrize("B,N,S,P", [(1, 1, 262_145, 37), (1, 2, 70_001, 3), (3, 5, 40_000, 1)])
def test_a_choice_out_of_range_marks_its_source_wherever_it_is(B, N, S, P):
    """Few sources with many choices are counted by several CTAs each; the choice that is wrong is in the share of a later one."""
    E = N * P
    experts = np.random.default_rng(S).integers(-1, E, (B, N, S)).astype(np.int32)
    for at, value in ((S - 1, E), (S // 2 + 5, -2), (0, 2 ** 31 - 1)):
        wrong = experts.copy()
        wrong[B - 1, N - 1, at] = value
        r = ms.route_demand(dev(wrong), E)
        wrong[B - 1, N - 1, at] = -1
        status = r["status"].cpu().numpy()
        assert status[B - 1, N - 1] == ms.ST_BAD_INPUT and (status.reshape(-1)[:-1] == 0).all()
        for k, v in zip(("demand", "counts", "slot"), plain_route(wrong, E)):
            assert (r[k].cpu().numpy() == v).all(), k
