"""The experts' feed-forward block, its gradients and the 4-bit products against 64-bit arithmetic, with bounds counted operation
by operation: half a step of the type (finfo.eps / 2) for every rounding to it, n steps of 2^-23 of the sum of
magnitudes for a sum of n products in 32 bits (each addition may cut instead of round)."""
import math

import pytest
import torch

import paper_2605_26845_b200 as ms
from paper_2605_26845_b200.workload import random_matrices

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
F32 = 2.0 ** -20        # relative error of an activation, and of the few products around it, in 32 bits
SLOPE, CURVE = 1.13, 0.81     # bounds of |act'| and |act''| of both activations


def gamma(n):
    return (n + 16) * 2.0 ** -23


class Rounded:
    """Half a step of the type at a value, and of its smallest numbers around 0."""
    def __init__(self, dtype):
        self.step = torch.finfo(dtype).eps / 2
        self.tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2

    def __call__(self, v, err):
        """Error of a value with error err after it has been rounded to the type."""
        return err + self.step * (v.abs() + err) + self.tiny


def act_of(a, kind):
    if kind == "silu":
        s = torch.sigmoid(a)
        return a * s, s + a * s * (1 - s)
    F = torch.special.ndtr(a)
    return a * F, F + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)


def spans(offsets, E):
    o = offsets.tolist()
    return [(g % E, slice(o[g], o[g + 1])) for g in range(len(o) - 1) if o[g] < o[g + 1]]


def forward(x, wg, wu, wd, kind, rnd):
    """a, u, y of one group's rows in 64 bits, each with its error."""
    D, I = wg.shape[1], wg.shape[0]
    a, u = x @ wg.T, x @ wu.T
    ea, eu = gamma(D) * (x.abs() @ wg.abs().T), gamma(D) * (x.abs() @ wu.abs().T)
    f, _ = act_of(a, kind)
    h = f * u
    eh = rnd(h, SLOPE * ea * (u.abs() + eu) + f.abs() * eu + F32 * (h.abs() + f.abs() * eu + SLOPE * ea * u.abs()) + F32 * a.abs() * u.abs())
    y = h @ wd.T
    ey = rnd(y, eh @ wd.abs().T + gamma(I) * ((h.abs() + eh) @ wd.abs().T))
    return (a, ea), (u, eu), (y, ey)          # (a and u are kept in 32 bits, as they are summed)


def backward(dy, x, a, u, wg, wu, wd, kind, rnd):
    """dx and the weights' gradients of one group's rows, from a and u with their errors; (value, error) each. Errors of the weights'
    sums leave out the rounding of the end: groups add up first."""
    D, I, R = wg.shape[1], wg.shape[0], x.shape[0]
    (a, ea), (u, eu) = a, u
    dh = dy @ wd
    edh = gamma(D) * (dy.abs() @ wd.abs())
    f, s = act_of(a, kind)
    ef, es = SLOPE * ea + F32 * a.abs(), CURVE * ea + F32 * (1 + a.abs())
    def times(p, ep, q, eq):
        return p * q, (ep * (q.abs() + eq) + p.abs() * eq) * (1 + F32) + F32 * (p * q).abs()
    h, eh = times(f, ef, u, eu)
    du, edu = times(dh, edh, f, ef)
    t, et = times(dh, edh, u, eu)
    da, eda = times(t, et, s, es)
    eh, edu, eda = rnd(h, eh), rnd(du, edu), rnd(da, eda)
    dx = da @ wg + du @ wu
    m = eda @ wg.abs() + edu @ wu.abs()
    edx = rnd(dx, m + gamma(2 * I) * (m + da.abs() @ wg.abs() + du.abs() @ wu.abs()))
    out = {}
    for k, (p, ep, q, eq) in dict(dw_gate=(da, eda, x, 0 * x), dw_up=(du, edu, x, 0 * x), dw_down=(dy, 0 * dy, h, eh)).items():
        e = ep.T @ (q.abs() + eq) + p.abs().T @ eq
        out[k] = (p.T @ q, e, p.abs().T @ q.abs() + e)
    return (dx, edx), out


def inputs(R, D, I, E, dtype, seed, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)
    return normal(R, D, std=scale), normal(E, I, D, std=D ** -0.5), normal(E, I, D, std=D ** -0.5), normal(E, D, I, std=I ** -0.5), normal(R, D)


def offsets_of(lengths, first=0):
    return torch.tensor([first] + lengths, dtype=torch.int32).cumsum(0).int().cuda()


def close(got, want, err, what):
    off = (got.double() - want).abs() - err
    assert torch.isfinite(got).all(), what
    assert (off <= 0).all(), (what, off.max().item(), (got.double() - want).abs().max().item())


def check(x, wg, wu, wd, dy, offsets, kind, train=True, same_rows=None):
    """same_rows: other offsets that give every expert the same rows, for the plain form."""
    E, dtype = wg.shape[0], x.dtype
    rnd = Rounded(dtype)
    R, D, I = x.shape[0], wg.shape[2], wg.shape[1]
    rows = torch.zeros(R, dtype=torch.bool, device="cuda")
    out, status = torch.full_like(x, 7.0), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    y, saved = ms.expert_ffn(x, wg, wu, wd, offsets, act=kind, save=True, out=out, status=status)
    assert status.item() == 0 and y is out
    assert torch.equal(ms.expert_ffn(x, wg, wu, wd, offsets, act=kind, out=torch.full_like(x, 7.0)), y)
    if train:
        into = dict(dx=torch.full_like(x, 7.0), dw_gate=torch.full_like(wg, 9.0), dw_up=torch.full_like(wu, 9.0), dw_down=torch.full_like(wd, 9.0))
        grads = ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved, act=kind, out=into, status=status)
        assert status.item() == 0
        total = {k: torch.zeros((3,) + tuple(grads[k].shape), dtype=torch.float64, device="cuda") for k in ("dw_gate", "dw_up", "dw_down")}
    count = [0] * E
    for e, s in spans(offsets if same_rows is None else same_rows, E):
        rows[s] = True
        count[e] += s.stop - s.start
        args = [t.double() for t in (x[s], wg[e], wu[e], wd[e])]
        a, u, (want, err) = forward(*args, kind, rnd)
        close(y[s], want, err, "y")
        close(saved["gate"][s], *a, "gate")
        close(saved["up"][s], *u, "up")
        if train:
            (dx, edx), parts = backward(dy[s].double(), args[0], a, u, *args[1:], kind, rnd)
            close(grads["dx"][s], dx, edx, "dx")
            for k, v in parts.items():
                for q in range(3):
                    total[k][q, e] += v[q]
    assert (y[~rows] == 7.0).all()
    if train:
        assert (grads["dx"][~rows] == 7.0).all()
        for k, (want, err, size) in total.items():
            for e in range(E):
                close(grads[k][e], want[e], rnd(want[e], err[e] + gamma(count[e]) * size[e]), k)
                assert count[e] or (grads[k][e] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R,D,I,lengths,E", [
    (1, 8, 8, [1], 1), (5, 16, 24, [0, 2, 3], 3), (37, 72, 200, [9, 0, 17, 11], 2), (64, 264, 136, [64], 1), (64, 128, 64, [1] * 64, 64),
    (12, 200, 72, [12], 1), (40, 72, 136, [33, 0, 0, 5, 0, 2, 0, 0], 8), (40, 1000, 264, [0, 1, 0, 9, 2, 3, 0, 25], 4)])
def test_few_rows(R, D, I, lengths, E, dtype):
    check(*inputs(R, D, I, E, TYPES[dtype], R + D), offsets_of(lengths), "silu")


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R,D,I,lengths,E", [
    (128, 64, 128, [128], 1), (129, 128, 256, [129], 1), (65, 8, 8, [65], 1), (200, 72, 40, [1, 127, 72], 3), (300, 200, 264, [0, 299, 0, 1], 4),
    (257, 1000, 136, [100, 7, 0, 50, 93, 7], 2), (400, 264, 520, [63, 64, 65, 66, 17, 15, 16, 94], 4), (3001, 512, 384, [1500, 1, 0, 1500], 2),
    (33, 1032, 1032, [0, 33], 2), (150, 2056, 712, [150], 1), (300, 1024, 520, [1, 128, 0, 171], 4), (100, 520, 1024, [60, 40], 1)])
def test_row_tiles(R, D, I, lengths, E, dtype, kind):
    check(*inputs(R, D, I, E, TYPES[dtype], R + I), offsets_of(lengths), kind)


def test_many_small_groups_of_many_experts():
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(0, 9, (40 * 6,), generator=g).tolist()
    check(*inputs(sum(lengths), 96, 80, 40, torch.bfloat16, 5), offsets_of(lengths), "silu")
    lengths = torch.randint(0, 2, (3 * 700,), generator=g).tolist()       # over a thousand groups
    check(*inputs(sum(lengths), 64, 64, 3, torch.float16, 6), offsets_of(lengths), "gelu")


def test_a_hundred_thousand_groups_of_one_expert():
    lengths = torch.randint(0, 2, (100000,), generator=torch.Generator().manual_seed(2)).tolist()
    R = sum(lengths)
    check(*inputs(R, 64, 72, 1, torch.bfloat16, 7), offsets_of(lengths), "silu", same_rows=offsets_of([R]))


@pytest.mark.parametrize("R", [40, 700])
def test_rows_outside_the_groups_are_neither_used_nor_written(R):
    x, wg, wu, wd, dy = inputs(R, 136, 72, 3, torch.bfloat16, 8)
    offsets = offsets_of([R // 3, 0, R // 3], first=5)
    for t in (x, dy):
        t[:5] = math.nan
        t[5 + 2 * (R // 3):] = math.inf
    check(x, wg, wu, wd, dy, offsets, "silu")


@pytest.mark.parametrize("R", [48, 600])
def test_a_row_that_is_not_finite_stays_among_its_own(R):
    x, wg, wu, wd, dy = inputs(R, 128, 136, 2, torch.bfloat16, 9)
    half = R // 2 - 3
    offsets = offsets_of([half, R - half])
    clean, saved = ms.expert_ffn(x, wg, wu, wd, offsets, save=True)
    grads = ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved)
    x[half - 1] = math.nan                                # the row before the other expert's first
    y, saved2 = ms.expert_ffn(x, wg, wu, wd, offsets, save=True)
    bad = ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved2)
    others = torch.arange(R, device="cuda") != half - 1
    assert torch.isnan(y[half - 1]).all() and torch.equal(y[others], clean[others])
    assert torch.isnan(bad["dx"][half - 1]).all() and torch.equal(bad["dx"][others], grads["dx"][others])
    for k in ("dw_gate", "dw_up", "dw_down"):
        assert torch.isnan(bad[k][0]).any() and torch.equal(bad[k][1], grads[k][1])


def test_large_values_saturate_the_activation():
    for dtype in TYPES.values():
        x, wg, wu, wd, dy = inputs(150, 64, 64, 1, dtype, 10, scale=30.0)
        for kind in ("silu", "gelu"):
            check(x, wg, wu, wd, dy, offsets_of([150]), kind)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("R", [9, 400])
def test_the_activations_tails_relative_to_themselves(R, kind):
    """With unit weights y = act(a) and dx = act'(a) of the numbers in x, each rounded twice; in 32 bits exp(-v) is off by 2 + 1.2 v
    steps of 2^-23, its argument by one, hence (2 + 2.2 * 41) * 2^-23 and a few more, below 2^-16."""
    n = 64
    a = torch.linspace(-9, 9, R * (n - 1), device="cuda").bfloat16().view(R, n - 1)
    a = a[torch.randperm(R, generator=torch.Generator().manual_seed(0)).cuda()]
    one = torch.ones((R, 1), dtype=torch.bfloat16, device="cuda")
    x, eye = torch.cat([a, one], 1), torch.eye(n, dtype=torch.bfloat16, device="cuda")[None].contiguous()
    wu = torch.zeros_like(eye)
    wu[0, :, n - 1] = 1                                   # u = 1; the last column of dx has the sums of du
    y, saved = ms.expert_ffn(x, eye, wu, eye, offsets_of([R]), act=kind, save=True)
    grads = ms.expert_ffn_backward(torch.ones_like(x), x, eye, wu, eye, offsets_of([R]), saved, act=kind)
    v = a.double()
    if kind == "gelu":                                    # (erfc: ndtr is 1 + erf, of which nothing is left in the tail)
        part = torch.special.erfc(-v / math.sqrt(2)) / 2, v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        f, s = v * part[0], part[0] + part[1]
    else:
        part = torch.sigmoid(v), v * torch.sigmoid(v) * torch.sigmoid(-v)
        f, s = v * part[0], part[0] + part[1]
    twice = 2 * (torch.finfo(torch.bfloat16).eps / 2) * 1.01 + 2.0 ** -16
    assert ((y[:, :-1].double() - f).abs() <= twice * f.abs()).all()
    # (the slope is a sum of two parts, each as near as that)
    assert ((grads["dx"][:, :-1].double() - s).abs() <= twice * s.abs() + 2.0 ** -16 * (part[0].abs() + part[1].abs())).all()


@pytest.mark.parametrize("R", [20, 300])
def test_offsets_out_of_order_are_reported(R):
    x, wg, wu, wd, dy = inputs(R, 64, 64, 2, torch.bfloat16, 11)
    saved = dict(gate=torch.zeros((R, 64), device="cuda"), up=torch.zeros((R, 64), device="cuda"))
    for bad in ([0, 9, 8], [-1, 3, R], [0, 5, R + 1], [3, 2, 1], [2 ** 31 - 1, -2 ** 31, 0]):
        offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ms.expert_ffn(x, wg, wu, wd, offsets, status=status)
        assert status.item() == ms.ST_BAD_INPUT
        status.zero_()
        ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved, status=status)
        assert status.item() == ms.ST_BAD_INPUT


def test_no_rows():
    x, wg, wu, wd, dy = inputs(0, 64, 72, 3, torch.bfloat16, 12)
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    y, saved = ms.expert_ffn(x, wg, wu, wd, offsets, save=True)
    grads = ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved)
    assert y.shape == (0, 64) and all((grads[k] == 0).all() for k in ("dw_gate", "dw_up", "dw_down"))
    x, _, _, _, dy = inputs(100, 64, 72, 3, torch.bfloat16, 12)           # rows, but no groups with any
    check(x, wg, wu, wd, dy, offsets, "silu")


def test_gradients_against_differences():
    """Central differences of sum(y dy) in 64 bits along random directions: the formulas themselves."""
    x, wg, wu, wd, dy = inputs(90, 64, 72, 2, torch.float16, 13)
    offsets = offsets_of([40, 50])
    def loss(p):
        return sum((act_of(p[0][s] @ p[1][e].T, "gelu")[0] * (p[0][s] @ p[2][e].T) @ p[3][e].T * dy[s].double()).sum() for e, s in spans(offsets, 2))
    _, saved = ms.expert_ffn(x, wg, wu, wd, offsets, act="gelu", save=True)
    grads = ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved, act="gelu")
    p = [t.double() for t in (x, wg, wu, wd)]
    for k, name in enumerate(("dx", "dw_gate", "dw_up", "dw_down")):
        d = torch.randn(p[k].shape, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(k))
        h = 1e-5
        up, down = [q.clone() for q in p], [q.clone() for q in p]
        up[k] += h * d
        down[k] -= h * d
        want = ((loss(up) - loss(down)) / (2 * h)).item()
        got = (grads[name].double() * d).sum().item()
        # every gradient value is off by a few half steps of its type, the difference by h^2 and what 64 bits lose
        bound = 6 * torch.finfo(x.dtype).eps / 2 * (grads[name].double().abs() * d.abs()).sum().item() + 1e-6 * abs(want) + 1e-5
        assert abs(got - want) <= bound, (name, got, want, bound)


def quantised(E, N, K, group, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    q = torch.randint(0, 256, (E, N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scale = (torch.rand((E, N, K // group), generator=g, device="cuda") * 0.2 - 0.1).to(dtype)
    w = torch.stack([q % 16, q // 16], -1).double().view(E, N, K // group, group) - 8
    return q, scale, (w * scale.double()[..., None]).view(E, N, K)


@pytest.mark.parametrize("gated", [None, "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R,K,N,group,lengths,E", [
    (1, 32, 1, 32, [1], 1), (1, 128, 16, 128, [0, 1, 0], 3), (7, 96, 17, 32, [7], 1), (8, 192, 40, 64, [8], 1), (9, 1024, 33, 128, [4, 0, 5, 0], 2), (23, 320, 200, 64, [23], 1),
    (61, 2048, 264, 64, [1] * 20 + [41] + [0] * 11, 32), (50, 160, 48, 32, [5, 20, 0, 25], 2), (3, 7168, 520, 128, [1, 1, 1], 3), (40, 256, 24, 128, [1, 2] * 13 + [1, 0], 2)])
def test_products_with_4_bit_weights(R, K, N, group, lengths, E, dtype, gated):
    dtype = TYPES[dtype]
    rnd = Rounded(dtype)
    x = torch.randn((R, K), generator=torch.Generator("cuda").manual_seed(R), device="cuda").to(dtype)
    q, scale, w = quantised(E, N, K, group, dtype, N)
    up = quantised(E, N, K, group, dtype, N + 1) if gated else (None, None, None)
    offsets, status = offsets_of(lengths), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    out = torch.full((R, N), 7.0, dtype=dtype, device="cuda")
    y = ms.expert_matvec4(x, q, scale, offsets, up[0], up[1], act=gated or "silu", out=out, status=status)
    assert status.item() == 0 and y is out
    for e, s in spans(offsets, E):
        v = x[s].double()
        want, err = v @ w[e].T, gamma(K) * (v.abs() @ w[e].abs().T)
        if gated:
            u, eu = v @ up[2][e].T, gamma(K) * (v.abs() @ up[2][e].abs().T)
            f, _ = act_of(want, gated)
            err = SLOPE * err * (u.abs() + eu) + f.abs() * eu + F32 * (f * u).abs() + F32 * want.abs() * u.abs()
            want = f * u
        close(y[s], want, rnd(want, err), "y")
    for bad in ([1, 0, R], [0, 0, R + 1]):
        if E == 1 or E == 2:
            o = torch.tensor(bad, dtype=torch.int32, device="cuda")
            ms.expert_matvec4(x, q, scale, o, up[0], up[1], out=out, status=status)
            assert status.item() == ms.ST_BAD_INPUT


def test_4_bit_rows_outside_the_groups_are_neither_used_nor_written():
    x = torch.full((30, 256), math.nan, dtype=torch.bfloat16, device="cuda")
    x[4:19] = 1.0
    q, scale, w = quantised(2, 40, 256, 64, torch.bfloat16, 3)
    y = ms.expert_matvec4(x, q, scale, offsets_of([6, 9], first=4), out=torch.full((30, 40), 7.0, dtype=torch.bfloat16, device="cuda"))
    assert (y[:4] == 7).all() and (y[19:] == 7).all() and torch.isfinite(y).all()


def test_from_the_routers_choices_to_the_layers_output():
    """Choices to demand, schedule, places, and the experts on what every rank received, against the layer computed token by token; then
    the same with the batch of one matching alone, and the gradients of the experts' inputs."""
    N, P, T, top, D, I = 4, 2, 60, 2, 64, 72
    E, dtype = N * P, torch.bfloat16
    g = torch.Generator("cuda").manual_seed(3)
    tokens = torch.randn((N, T, D), generator=g, device="cuda").to(dtype)
    chosen = torch.rand((N, T, E), generator=g, device="cuda").topk(top).indices.int()
    chosen[0, :5] = -1
    r = ms.route_demand(chosen.view(1, N, T * top).contiguous(), E)
    schedule = ms.mw_decompose(r["demand"], 2 * N)
    slots = ms.schedule_slots(r["demand"], schedule.perm, schedule.dur, schedule.count, r["counts"])
    assert (schedule.status == 0).all() and (slots["status"] == 0).all()
    _, wg, wu, wd, _ = inputs(1, D, I, E, dtype, 4)
    # send buffers, by expert
    slot = r["slot"][0].long()
    sent = [int(v) for v in (slot >= 0).sum(1)]
    send = [torch.empty((n, D), dtype=dtype, device="cuda") for n in sent]
    for i in range(N):
        s = torch.nonzero(slot[i] >= 0)[:, 0]
        send[i][slot[i][s]] = tokens[i][s // top]
    first = torch.cumsum(r["demand"][0].long(), 1) - r["demand"][0].long()        # of a pair, in the source's buffer
    # transfers, matching by matching
    recv = [torch.full((int(slots["rows"][0, j]), D), math.nan, dtype=dtype, device="cuda") for j in range(N)]
    moves = []
    for k in range(int(schedule.count[0])):
        for i in range(N):
            j, n = int(schedule.perm[0, k, i]), int(slots["length"][0, k, i])
            a, b = int(first[i, j] + slots["start"][0, k, i]), int(slots["row"][0, k, i])
            recv[j][b:b + n] = send[i][a:a + n]
            moves.append((i, j, a, b, n))
    back = [torch.full((n, D), math.nan, dtype=dtype, device="cuda") for n in sent]
    for j in range(N):
        mine = slice(j * P, (j + 1) * P)
        weights = [w[mine].contiguous() for w in (wg, wu, wd)]
        offsets = slots["offsets"][0, j]
        y = ms.expert_ffn(recv[j], *weights, offsets)
        k = int(torch.diff(offsets[::P]).argmax())                                   # one matching alone: the same rows
        part = ms.expert_ffn(recv[j], *weights, offsets[k * P:(k + 1) * P + 1].contiguous(), out=torch.zeros_like(y))
        rows = slice(int(offsets[k * P]), int(offsets[(k + 1) * P]))
        assert (part[:rows.start] == 0).all() and (part[rows.stop:] == 0).all()
        assert (part[rows].float() - y[rows].float()).abs().max() <= 2.0 ** -6 * y[rows].float().abs().max()
        for i, to, a, b, n in moves:
            if to == j:
                back[i][a:a + n] = y[b:b + n]
    rnd = Rounded(dtype)
    for i in range(N):
        for t in range(T):
            for c in range(top):
                e, at = int(chosen[i, t, c]), int(slot[i, t * top + c])
                if e < 0:
                    continue
                _, _, (want, err) = forward(tokens[i, t:t + 1].double(), wg[e].double(), wu[e].double(), wd[e].double(), "silu", rnd)
                close(back[i][at:at + 1], want, err, (i, t, c))


def test_replayed_from_graphs_and_on_two_streams_at_once():
    x, wg, wu, wd, dy = inputs(500, 128, 136, 2, torch.bfloat16, 20)
    offsets = offsets_of([200, 300])
    y, saved = ms.expert_ffn(x, wg, wu, wd, offsets, save=True)
    want = ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved)
    graphs, results = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y2, saved2 = ms.expert_ffn(x, wg, wu, wd, offsets, save=True)
            results.append((y2, ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved2)))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, graph in zip(streams, graphs):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(5):
                graph.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = [ms.expert_ffn(x, wg, wu, wd, offsets) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(e, y) for e in eager)
    for y2, grads in results:
        assert torch.equal(y2, y) and all(torch.equal(grads[k], want[k]) for k in want)      # the same bits every time


def test_schedules_offsets_of_a_random_demand():
    D = random_matrices(1, 6, seed=4, kind="uniform", high=90)
    d = torch.from_numpy(D).cuda()
    counts = torch.stack([d // 3, d - d // 3], -1).view(1, 6, 12).contiguous()
    s = ms.mw_decompose(d, 40)
    slots = ms.schedule_slots(d, s.perm, s.dur, s.count, counts)
    for j in (0, 5):
        R = int(slots["rows"][0, j])
        check(*inputs(R, 72, 64, 2, torch.bfloat16, j), slots["offsets"][0, j], "silu")


def test_probed_experts_make_a_model_that_schedules_are_scored_with():
    _, wg, wu, wd, _ = inputs(1, 256, 128, 2, torch.bfloat16, 30)
    pairs = [quantised(2, n, k, 64, torch.bfloat16, n)[:2] for n, k in ((128, 256), (128, 256), (256, 128))]
    d = torch.from_numpy(random_matrices(2, 8, seed=1, high=500)).cuda()
    s = ms.mw_decompose(d, 8)
    for weights in ((wg, wu, wd), pairs):
        probe = ms.probe_expert(weights, tokens=(1, 8, 300), base=dict(ms.DEFAULT_MODEL, reconfig_ns=7), reps=3)
        m = probe["model"]
        assert probe["tokens"] == [1, 8, 300] and len(probe["ns"]) == 3 and min(probe["ns"]) > 0
        assert m["bytes_per_token"] == 512 and m["reconfig_ns"] == 7 and m["expert_fixed_ns"] > 0
        assert m["expert_ps_per_token"] >= 0 and m["expert_knee_tokens"] in (1, 8, 300)
        score = ms.schedule_eval(d, s.perm, s.dur, s.count, m)
        assert (score["status"] == 0).all() and (score["makespan_overlap_ns"] >= m["expert_fixed_ns"]).all()
    with pytest.raises(ms.MoeschedError):
        ms.probe_expert((wg, wu, wd), tokens=(0, 4))


def test_two_experts_layers_in_4_bits():
    """An expert in 4 bits is two calls: gate and up with the activation, then down."""
    dtype, E, D, I = torch.float16, 3, 192, 128
    rnd = Rounded(dtype)
    x = torch.randn((11, D), generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(dtype)
    g, u, w = quantised(E, I, D, 64, dtype, 1), quantised(E, I, D, 64, dtype, 2), quantised(E, D, I, 32, dtype, 3)
    offsets = offsets_of([2, 9, 0])
    h = ms.expert_matvec4(x, g[0], g[1], offsets, u[0], u[1], act="gelu")
    y = ms.expert_matvec4(h, w[0], w[1], offsets)
    for e, s in spans(offsets, E):
        a, b = x[s].double() @ g[2][e].T, x[s].double() @ u[2][e].T
        ea, eb = gamma(D) * (x[s].double().abs() @ g[2][e].abs().T), gamma(D) * (x[s].double().abs() @ u[2][e].abs().T)
        f, _ = act_of(a, "gelu")
        v = f * b
        ev = rnd(v, SLOPE * ea * (b.abs() + eb) + f.abs() * eb + F32 * (v.abs() + a.abs() * b.abs()))
        want = v @ w[2][e].T
        close(y[s], want, rnd(want, ev @ w[2][e].abs().T + gamma(I) * ((v.abs() + ev) @ w[2][e].abs().T)), "y")


@pytest.mark.parametrize("E,per", [(600, 1), (1024, 1), (1024, 2)])
def test_as_many_experts_as_there_may_be(E, per):
    g = torch.Generator().manual_seed(E)
    lengths = torch.randint(0, 3, (E * per,), generator=g).tolist()
    R = sum(lengths)
    assert R <= 4 * E + 8                                 # the few-row kernel; and below row tiles of the same
    data = inputs(R, 72, 24, E, torch.bfloat16, E)
    check(*data, offsets_of(lengths), "silu")
    x, wg, wu, wd, dy = inputs(5 * E, 72, 24, E, torch.bfloat16, E)
    lengths = [0] * E
    lengths[E - 1], lengths[3] = 3 * E, 2 * E
    check(x, wg, wu, wd, dy, offsets_of(lengths), "silu", train=False)
    q, scale, w = quantised(E, 24, 64, 32, torch.bfloat16, E)
    v = x[:R, :64].contiguous()
    lengths = torch.randint(0, 3, (E * per,), generator=torch.Generator().manual_seed(E)).tolist()
    y = ms.expert_matvec4(v, q, scale, offsets_of(lengths))
    rnd = Rounded(torch.bfloat16)
    for e, s in spans(offsets_of(lengths), E)[::37]:
        want = v[s].double() @ w[e].T
        close(y[s], want, rnd(want, gamma(64) * (v[s].double().abs() @ w[e].abs().T)), "y")
