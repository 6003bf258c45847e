"""What the experts' entry points refuse, without a GPU."""
import pytest
import torch

import __graft_entry__ as entry
import paper_2605_26845_b200 as ms


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return ms.load_library()


A = [1 << 20 | 4096 * k for k in range(16)]      # addresses that are never followed


def with_changes(names, at):
    p = dict(zip(names, A))
    p.update(at)
    return [p[n] for n in names]


def test_expert_ffn_checks_its_arguments(lib):
    names = ("x", "w_gate", "w_up", "w_down", "offsets", "y", "gate", "up", "scratch", "status")

    def call(R=10, D=64, I=72, E=2, groups=4, dtype=0, act=0, **at):
        return lib.moesched_expert_ffn(R, D, I, E, groups, dtype, act, *with_changes(names, at), None)

    for bad in (dict(R=-1), dict(D=0), dict(D=60), dict(D=65544), dict(I=4), dict(I=70), dict(E=0), dict(E=1025, groups=1025), dict(groups=0), dict(groups=3),
                dict(groups=1 << 25), dict(dtype=2), dict(dtype=-1), dict(act=2)):
        assert call(**bad) == -1, bad
    for n in names:
        assert call(**{n: None}) == -1, n                    # (gate and up: only both)
        assert call(**{n: A[0] + (2 if n in ("offsets", "status") else 8)}) == -1, n
    assert call(scratch=A[8] + 128) == -1


def test_expert_ffn_backward_checks_its_arguments(lib):
    names = ("dy", "x", "w_gate", "w_up", "w_down", "offsets", "gate", "up", "dx", "dw_gate", "dw_up", "dw_down", "scratch", "status")

    def call(R=10, D=64, I=72, E=2, groups=4, dtype=0, act=0, **at):
        return lib.moesched_expert_ffn_backward(R, D, I, E, groups, dtype, act, *with_changes(names, at), None)

    for bad in (dict(R=-1), dict(D=60), dict(I=70), dict(E=0), dict(groups=3), dict(dtype=2), dict(act=-1)):
        assert call(**bad) == -1, bad
    for n in names:
        assert call(**{n: None}) == -1, n
        assert call(**{n: A[0] + (2 if n in ("offsets", "status") else 8)}) == -1, n
    assert call(R=0, dw_up=None) == -1


def test_expert_matvec4_checks_its_arguments(lib):
    names = ("x", "w", "scale", "w_up", "scale_up", "offsets", "y", "status")

    def call(R=10, K=128, N=30, E=2, groups=4, group=64, dtype=0, act=0, **at):
        return lib.moesched_expert_matvec4(R, K, N, E, groups, group, dtype, act, *with_changes(names, at), None)

    for bad in (dict(R=-1), dict(K=0), dict(K=96), dict(N=0), dict(E=0), dict(groups=3), dict(group=16), dict(group=48), dict(group=0), dict(dtype=2), dict(act=2)):
        assert call(**bad) == -1, bad
    for n in names:
        assert call(**{n: None}) == -1, n                    # (w_up and scale_up: only both)
        assert call(**{n: A[0] + (2 if n in ("offsets", "status") else 8)}) == -1, n


def test_scratch_sizes(lib):
    plan = lambda R, groups: -(-16 * (R // 128 + groups + 1) // 256) * 256    # noqa: E731
    assert ms.expert_scratch_bytes(1000, 64, 4) == plan(1000, 4) + 128000
    assert ms.expert_scratch_bytes(1000, 64, 4, True) == plan(1000, 4) + 3 * 128000
    assert ms.expert_scratch_bytes(-1, 64, 4) == ms.expert_scratch_bytes(10, 60, 4) == ms.expert_scratch_bytes(10, 64, 0) == 0


def test_the_binding_refuses_wrong_tensors(lib):
    x, w = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros((1, 8, 8), dtype=torch.bfloat16)
    o = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: ms.expert_ffn(x, w, w, w, o), lambda: ms.expert_ffn(x.float(), w, w, w, o), lambda: ms.expert_ffn(x, None, w, w, o),
                 lambda: ms.expert_ffn_backward(x, x, w, w, w, o, dict(gate=x, up=x)),
                 lambda: ms.expert_matvec4(x, w.byte(), w, o), lambda: ms.expert_matvec4(x, None, w, o)):
        with pytest.raises(ms.MoeschedError):
            call()


def test_more_rows_and_groups_than_are_numbered(lib):
    for rows, groups in (((1 << 30) + 1, 4), (1 << 31, 4), ((1 << 32) + 10, 4), (10, (1 << 24) + 4), (10, (1 << 32) + 4)):
        assert ms.expert_scratch_bytes(rows, 64, groups) == 0, (rows, groups)
    assert ms.expert_scratch_bytes(1 << 30, 8, 1 << 24) > 0

    class Rows(torch.Tensor):                              # says that it is on a GPU; nothing is read
        is_cuda = True

    def rows(shape, dtype):                                # of that shape, and dense where it counts
        t = torch.empty(0, dtype=dtype).as_subclass(Rows)
        t.__class__ = type("Big", (Rows,), {"shape": torch.Size(shape), "dim": lambda s: len(shape), "is_contiguous": lambda s: True,
                                            "numel": lambda s: torch.Size(shape).numel(), "dtype": dtype})
        return t

    offsets = rows((3,), torch.int32)
    assert ms._expert_rows(rows((1 << 30, 8), torch.bfloat16), offsets, 2) == (0, 2)
    for x, o in ((rows(((1 << 30) + 1, 8), torch.bfloat16), offsets), (rows(((1 << 32) + 5, 8), torch.bfloat16), offsets),
                 (rows((5, 8), torch.bfloat16), rows(((1 << 32) + 3,), torch.int32))):
        with pytest.raises(ms.MoeschedError, match="2\\^30"):
            ms._expert_rows(x, o, 2)


def test_tensors_that_want_a_gradient_are_refused_where_autograd_records():
    x, w = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros((1, 8, 8), dtype=torch.bfloat16)
    o, q = torch.zeros(2, dtype=torch.int32), torch.zeros((1, 8, 4), dtype=torch.uint8)

    def calls(x, w, dy, s):
        return (lambda: ms.expert_ffn(x, w, w.detach(), w.detach(), o), lambda: ms.expert_ffn_backward(dy, x, w.detach(), w, w.detach(), o, {}),
                lambda: ms.expert_matvec4(x, q, s, o), lambda: ms.expert_matvec4(x, q, s.detach(), o, q, s))

    want, wide = (t.clone().requires_grad_() for t in (x, w))
    for call in calls(want, w, x, w) + calls(x, wide, x, wide):
        with pytest.raises(ms.MoeschedError, match="no_grad"):
            call()
        with torch.no_grad(), pytest.raises(ms.MoeschedError, match="CUDA tensor"):       # (the next check)
            call()
    for call in calls(x, w, x, w):
        with pytest.raises(ms.MoeschedError, match="CUDA tensor"):
            call()
    with pytest.raises(ms.MoeschedError, match="no_grad"):
        ms.expert_ffn(x, w, w, w, o, out=want)
    with pytest.raises(ms.MoeschedError, match="no_grad"):
        ms.expert_ffn_backward(want, x, w, w, w, o, {})


def test_the_curve_through_measured_times():
    tokens = [1, 16, 64, 256, 1024, 4096]
    for fixed, slope, knee in ((100.0, 0.25, 64), (7.5, 0.0, 4096), (31.0, 3.0, 1)):          # its own curve is found again
        times = [fixed + max(0, g - knee) * slope for g in tokens]
        got = ms._expert_curve(tokens, times)
        assert all(abs(got[0] + max(0, g - got[2]) * got[1] - t) <= 1e-9 * t for g, t in zip(tokens, times)), got
    # four experts, of which one token meets only one: the curve is not laid through that one, with the others at a third of their times
    times = [24.8, 69.6, 70.3, 72.5, 84.0, 227.5]
    fixed, slope, knee = ms._expert_curve(tokens, times)
    assert all(0.5 <= (fixed + max(0, g - knee) * slope) / t <= 2 for g, t in zip(tokens, times))
