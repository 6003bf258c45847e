"""What the entry points for tokens (norm, choice, rows and back) refuse, without a GPU."""
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


def test_rms_norm_checks_its_arguments(lib):
    names = ("x", "residual", "weight", "sum", "y", "q", "scale", "rstd")

    def call(rows=10, D=64, dtype=0, eps=1e-6, group=64, **at):
        return lib.moesched_rms_norm(rows, D, dtype, eps, group, *with_changes(names, at), None)

    for bad in (dict(rows=-1), dict(rows=(1 << 30) + 1), dict(D=0), dict(D=60), dict(D=65544), dict(dtype=3), dict(dtype=-1), dict(eps=-1e-9),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(group=0), dict(group=16), dict(group=96), dict(group=256)):
        assert call(**bad) == -1, bad
    for n in ("x", "residual", "weight", "sum", "q", "scale"):
        assert call(**{n: None}) == -1, n                    # (residual and sum, q and scale: only both)
    assert call(y=None, q=None, scale=None) == -1
    for n in names:
        assert call(**{n: A[0] + (2 if n == "rstd" else 8)}) == -1, n
    assert call(rows=0, x=None) == 0


def test_rms_norm_backward_checks_its_arguments(lib):
    names = ("dy", "h", "weight", "rstd", "dsum", "dx", "dweight", "scratch")

    def call(rows=10, D=64, dtype=0, **at):
        return lib.moesched_rms_norm_backward(rows, D, dtype, *with_changes(names, at), None)

    for bad in (dict(rows=-1), dict(D=12), dict(dtype=3), dict(rows=0, dweight=None)):
        assert call(**bad) == -1, bad
    for n in names:
        assert n == "dsum" or call(**{n: None}) == -1, n
        assert call(**{n: A[0] + (2 if n == "rstd" else 8)}) == -1, n
    assert ms.norm_scratch_bytes(10, 64) == 10 * 64 * 4 and ms.norm_scratch_bytes(1 << 20, 4096) == 148 * 4096 * 4 and ms.norm_scratch_bytes(1000, 16384) == (148 * 16384 + 1000) * 4
    assert ms.norm_scratch_bytes(-1, 64) == ms.norm_scratch_bytes(10, 60) == ms.norm_scratch_bytes((1 << 30) + 1, 64) == ms.norm_scratch_bytes((1 << 32) + 1, 64) == 0


def test_route_choose_checks_its_arguments(lib):
    for fn, names, needed in ((lib.moesched_route_choose, ("logits", "bias", "experts", "weights"), ("logits", "experts", "weights")),
                              (lib.moesched_route_choose_backward, ("dweights", "logits", "experts", "dlogits"), ("dweights", "logits", "experts", "dlogits"))):
        def call(rows=10, E=64, k=8, dtype=2, score=0, normalise=1, factor=1.0, **at):
            return fn(rows, E, k, dtype, score, normalise, factor, *with_changes(names, at), None)

        for bad in (dict(rows=-1), dict(rows=(1 << 30) + 1), dict(E=0), dict(E=1025), dict(k=0), dict(k=33), dict(E=7), dict(dtype=3), dict(score=2), dict(score=-1),
                    dict(factor=float("nan")), dict(factor=float("inf")), dict(factor=-float("inf"))):
            assert call(**bad) == -1, bad
        for n in needed:
            assert call(**{n: None}) == -1, n
        for n in names:
            assert call(**{n: A[0] + 2}) == -1 and call(**{n: A[0] + 1}) == -1, n
            assert call(dtype=0, **{n: A[0] + 1}) == -1, n
        assert call(rows=0, **{needed[0]: None}) == 0


def test_rows_check_their_arguments(lib):
    sends = ("x", "scale", "slot", "rows", "row_scale")
    backs = ("rows", "slot", "weights", "add", "y")
    grads = ("dy", "rows", "slot", "weights", "drows", "dweights")

    def send(G=2, T=10, k=3, row_bytes=64, scales=2, **at):
        return lib.moesched_tokens_to_rows(G, T, k, row_bytes, scales, *with_changes(sends, at), None)

    def back(G=2, T=10, k=3, D=64, dtype=0, **at):
        return lib.moesched_rows_to_tokens(G, T, k, D, dtype, *with_changes(backs, at), None)

    def grad(G=2, T=10, k=3, D=64, dtype=0, **at):
        return lib.moesched_rows_to_tokens_backward(G, T, k, D, dtype, *with_changes(grads, at), None)

    for call in (send, back, grad):
        for bad in (dict(G=-1), dict(T=-1), dict(G=1 << 20, T=1 << 11), dict(k=0), dict(k=33), dict(T=1 << 28, k=8, G=1)):
            assert call(**bad) == -1, (call, bad)
        assert call(G=0) == 0 and call(T=0) == 0
    for bad in (dict(row_bytes=0), dict(row_bytes=12), dict(row_bytes=(1 << 18) + 8), dict(scales=-1), dict(scales=65537), dict(scales=0)):
        assert send(**bad) == -1, bad
    for call in (back, grad):
        for bad in (dict(D=0), dict(D=12), dict(D=65544), dict(dtype=3), dict(dtype=-1)):
            assert call(**bad) == -1, bad
    for call, names, four, free in ((send, sends, ("slot",), ()), (back, backs, ("slot", "weights"), ("weights", "add")), (grad, grads, ("slot", "weights", "dweights"), ())):
        for n in names:
            assert n in free or call(**{n: None}) == -1, n
            assert call(**{n: A[0] + (2 if n in four else 8)}) == -1, n
    assert send(scales=0, scale=None) == -1


def test_rows_widen_checks_its_arguments(lib):
    names = ("q", "scale", "y")

    def call(R=10, D=64, group=32, dtype=0, **at):
        return lib.moesched_rows_widen(R, D, group, dtype, *with_changes(names, at), None)

    for bad in (dict(R=-1), dict(R=(1 << 30) + 1), dict(D=60), dict(group=0), dict(group=48), dict(dtype=3)):
        assert call(**bad) == -1, bad
    for n in names:
        assert call(**{n: None}) == -1 and call(**{n: A[0] + 8}) == -1, n
    assert call(R=0, q=None) == 0


def refused(on):
    """Calls with something wrong, on tensors made by on(shape, dtype); and with something missing."""
    i32, f32, f8 = torch.int32, torch.float32, torch.float8_e4m3fn

    def t(*shape, dtype=torch.bfloat16):
        return on(shape, dtype)

    x, w, slot, wide = t(6, 64), t(64), t(12, dtype=i32), t(6, 64, dtype=f32)
    rows, weights = t(12, 64), t(12, dtype=f32)
    l, ex = t(6, 10, dtype=f32), t(12, dtype=i32)
    rstd, q, s = t(6, dtype=f32), t(6, 64, dtype=f8), t(6, 2, dtype=f32)
    wrong = (
        lambda: ms.rms_norm(x, t(64, dtype=f32)), lambda: ms.rms_norm(x, t(32)), lambda: ms.rms_norm(w, x), lambda: ms.rms_norm(t(), w),
        lambda: ms.rms_norm(t(6, 60), t(60)), lambda: ms.rms_norm(t(6, 65544), t(65544)), lambda: ms.rms_norm(x.double(), w.double()), lambda: ms.rms_norm(x.t(), t(6)),
        lambda: ms.rms_norm(t(64, 8).t(), w), lambda: ms.rms_norm(x, t(128)[::2]),
        lambda: ms.rms_norm(x, w, eps=-1.0), lambda: ms.rms_norm(x, w, eps=float("nan")), lambda: ms.rms_norm(x, w, eps=float("inf")), lambda: ms.rms_norm(x, w, group=16),
        lambda: ms.rms_norm(x, w, want_y=False), lambda: ms.rms_norm(x, w, residual=t(5, 64)), lambda: ms.rms_norm(x, w, residual=wide),
        lambda: ms.rms_norm_backward(x, x, w, t(5, dtype=f32)), lambda: ms.rms_norm_backward(x, x, w, t(6)), lambda: ms.rms_norm_backward(wide, x, w, rstd),
        lambda: ms.rms_norm_backward(x, x, w, rstd, dsum=wide), lambda: ms.rms_norm_backward(x, x, w, rstd, scratch=t(8, dtype=torch.uint8)),
        lambda: ms.rms_norm_backward(x, x, w, rstd, scratch=t(1 << 16, dtype=f32)),
        lambda: ms.route_choose(l, 0), lambda: ms.route_choose(l, 11), lambda: ms.route_choose(l, 1 << 40), lambda: ms.route_choose(l, -1), lambda: ms.route_choose(l, 2, score="tanh"),
        lambda: ms.route_choose(l, 2, score=None), lambda: ms.route_choose(l.double(), 2), lambda: ms.route_choose(t(6, 0, dtype=f32), 1),
        lambda: ms.route_choose(t(6, 1025, dtype=f32), 2), lambda: ms.route_choose(t(6, 64, dtype=f32), 33), lambda: ms.route_choose(t(10, dtype=f32), 2),
        lambda: ms.route_choose(l, 2, bias=t(9, dtype=f32)), lambda: ms.route_choose(l, 2, bias=t(10)), lambda: ms.route_choose(l, 2, factor=float("inf")), lambda: ms.route_choose(l.t(), 2),
        lambda: ms.route_choose_backward(t(11, dtype=f32), l, ex), lambda: ms.route_choose_backward(weights, l, t(11, dtype=i32)), lambda: ms.route_choose_backward(weights, l, t(6, 2, dtype=i32)),
        lambda: ms.route_choose_backward(weights, l, t(0, dtype=i32)), lambda: ms.route_choose_backward(t(12), l, ex), lambda: ms.route_choose_backward(weights, l[0], ex),
        lambda: ms.tokens_to_rows(x, t(13, dtype=i32)), lambda: ms.tokens_to_rows(x, t(0, dtype=i32)), lambda: ms.tokens_to_rows(x, slot.long()), lambda: ms.tokens_to_rows(w, slot),
        lambda: ms.tokens_to_rows(x, t(6 * 33, dtype=i32)), lambda: ms.tokens_to_rows(x, t(1, 12, dtype=i32)), lambda: ms.tokens_to_rows(t(6, 12), slot),
        lambda: ms.tokens_to_rows(x.double(), slot), lambda: ms.tokens_to_rows(x, slot, scale=t(5, 2, dtype=f32)), lambda: ms.tokens_to_rows(x, slot, scale=t(6, 2)),
        lambda: ms.tokens_to_rows(x, slot, scale=t(6, 0, dtype=f32)), lambda: ms.tokens_to_rows(x, slot, scale=t(6, 65, dtype=f32)), lambda: ms.tokens_to_rows(x, slot, out_scale=s),
        lambda: ms.rows_to_tokens(rows, slot, 5), lambda: ms.rows_to_tokens(rows, slot, 0), lambda: ms.rows_to_tokens(rows, slot, 36), lambda: ms.rows_to_tokens(rows, t(10, dtype=i32), 2),
        lambda: ms.rows_to_tokens(rows, slot, 2, weights=t(12)), lambda: ms.rows_to_tokens(rows, slot, 2, add=rows), lambda: ms.rows_to_tokens(t(12, 64, dtype=f8), slot, 2),
        lambda: ms.rows_to_tokens(rows, t(12), 2),
        lambda: ms.rows_to_tokens_backward(x, x, slot, weights), lambda: ms.rows_to_tokens_backward(wide, rows, slot, weights), lambda: ms.rows_to_tokens_backward(x, rows, slot, t(12)),
        lambda: ms.rows_widen(x, s, 32), lambda: ms.rows_widen(q, s, 64), lambda: ms.rows_widen(q, s, 32, torch.float64), lambda: ms.rows_widen(q, s, 48), lambda: ms.rows_widen(q, s, 32, None),
    )
    missing = (
        lambda: ms.rms_norm(None, w), lambda: ms.rms_norm(x, None), lambda: ms.rms_norm_backward(None, x, w, rstd), lambda: ms.rms_norm_backward(x, x, w, None),
        lambda: ms.route_choose(None, 2), lambda: ms.route_choose_backward(weights, None, ex), lambda: ms.route_choose_backward(weights, l, None), lambda: ms.route_choose_backward(None, l, ex),
        lambda: ms.tokens_to_rows(None, slot), lambda: ms.tokens_to_rows(x, None), lambda: ms.rows_to_tokens(None, slot, 2), lambda: ms.rows_to_tokens(rows, None, 2),
        lambda: ms.rows_to_tokens_backward(x, rows, slot, None), lambda: ms.rows_widen(None, s, 32), lambda: ms.rows_widen(q, None, 32), lambda: ms.rms_norm([1.0], w),
    )
    right = (
        lambda: ms.rms_norm(x, w, residual=x, group=32), lambda: ms.rms_norm_backward(x, x, w, rstd), lambda: ms.route_choose(l, 2), lambda: ms.route_choose_backward(weights, l, ex),
        lambda: ms.tokens_to_rows(x, slot), lambda: ms.rows_to_tokens(rows, slot, 2), lambda: ms.rows_to_tokens_backward(x, rows, slot, weights), lambda: ms.rows_widen(q, s, 32),
    )
    return wrong, missing, right


def test_the_binding_refuses_wrong_tensors(lib):
    wrong, missing, right = refused(lambda shape, dtype: torch.zeros(shape, dtype=dtype))
    for n, call in enumerate(wrong):
        with pytest.raises(ms.MoeschedError, match="^(?!.*CUDA tensor)"):        # (something else than where the tensors are)
            call()
            print("not refused:", n)
    for call in missing + right:
        with pytest.raises(ms.MoeschedError, match="must be a CUDA tensor"):
            call()
    for call in (lambda: ms.route_choose(torch.zeros(4, 4), "two"), lambda: ms.rms_norm(torch.zeros(4, 8), torch.zeros(8), eps="no"),
                 lambda: ms._bound.rms_norm(1), lambda: ms._bound.bind(1)):
        with pytest.raises((TypeError, ValueError)):
            call()


def test_a_missing_part_of_the_binding_is_said(monkeypatch, lib):
    import sys
    monkeypatch.setattr(ms, "_bound", None)
    monkeypatch.delattr(ms, "_binding", raising=False)
    monkeypatch.setitem(sys.modules, ms.__name__ + "._binding", None)
    with pytest.raises(ms.MoeschedError, match="build"):
        ms.rms_norm(torch.zeros(4, 8), torch.zeros(8))


def test_tensors_that_want_a_gradient_are_refused_where_autograd_records(lib):
    x, w, slot = torch.zeros((4, 8)), torch.zeros(8), torch.zeros(8, dtype=torch.int32)
    want = x.clone().requires_grad_()
    f, r4 = torch.zeros(8), torch.zeros(4)
    calls = (lambda t: ms.rms_norm(t, w), lambda t: ms.rms_norm(x, w, residual=t), lambda t: ms.rms_norm_backward(t, x, w, r4),
             lambda t: ms.route_choose(t, 2), lambda t: ms.route_choose_backward(f, t, slot), lambda t: ms.tokens_to_rows(t, slot),
             lambda t: ms.rows_to_tokens(t, slot[:4], 2), lambda t: ms.rows_to_tokens(x, slot[:4], 2, add=t), lambda t: ms.rows_to_tokens_backward(t, torch.zeros((8, 8)), slot, f))
    for n, call in enumerate(calls):
        with pytest.raises(ms.MoeschedError, match="no_grad"):
            call(want)
        if n != 7:
            with torch.no_grad(), pytest.raises(ms.MoeschedError, match="CUDA tensor"):       # (the last check)
                call(want)
