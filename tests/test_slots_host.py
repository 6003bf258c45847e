"""What the entry points for demand and slots refuse, without a GPU."""
import pytest
import torch

import __graft_entry__ as entry
import paper_2605_26845_b200 as ms


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return ms.load_library()


A = [4096 * (k + 1) for k in range(12)]      # addresses that are never followed


def test_route_demand_checks_its_arguments(lib):
    def call(B=2, N=8, S=100, E=16, at=()):
        p = A[:5]
        for k, v in dict(at).items():
            p[k] = v
        return lib.moesched_route_demand(B, N, S, E, *p, None)

    for bad in (dict(B=-1), dict(N=0), dict(N=257, E=257), dict(S=-1), dict(E=7), dict(E=12), dict(E=1032), dict(B=1 << 30)):
        assert call(**bad) == -1, bad
    for k in range(5):
        assert call(at={k: None}) == -1 and call(at={k: A[k] + 2}) == -1, k
    assert call(B=0) == 0


def test_schedule_slots_checks_its_arguments(lib):
    def call(B=2, N=8, K=5, P=2, at=()):
        p = A[:12]
        for k, v in dict(at).items():
            p[k] = v
        return lib.moesched_schedule_slots(B, N, p[0], K, *p[1:4], P, *p[4:12], None)

    for bad in (dict(B=-1), dict(N=0), dict(N=257), dict(K=0), dict(P=0), dict(P=129)):
        assert call(**bad) == -1, bad
    for k in range(12):
        assert k == 10 or call(at={k: None}) == -1, k             # (no scratch is needed)
        assert k == 1 or call(at={k: A[k] + 2}) == -1, k
    assert lib.moesched_slots_scratch_bytes(2, 0, 5000) == lib.moesched_slots_scratch_bytes(-1, 8, 5000) == lib.moesched_slots_scratch_bytes(2, 8, 0) == 0
    assert lib.moesched_slots_scratch_bytes(2, 8, 30) == lib.moesched_slots_scratch_bytes(500, 8, 3000) == lib.moesched_slots_scratch_bytes(2, 129, 3000) == 0
    assert lib.moesched_slots_scratch_bytes(2, 8, 640) == 2 * 10 * 64 * 4
    assert call(B=0) == 0
    assert call(B=0, P=0, at={4: None, 9: None}) == 0


def test_the_binding_refuses_what_is_not_on_a_gpu(lib):
    with pytest.raises(ms.MoeschedError):
        ms.route_demand(torch.zeros((1, 2, 3), dtype=torch.int32), 4)
    with pytest.raises(ms.MoeschedError):
        ms.schedule_slots(*(torch.zeros(1, dtype=torch.int32) for _ in range(4)))
