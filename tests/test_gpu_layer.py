"""A layer as the operators make it together: norm, choice, demand, schedule, rows sent by its slots, the experts of every rank, rows back with their weights, and
the gradients of all of it, against the same layer in 64 bits with autograd."""
import pytest
import torch

import paper_2605_26845_b200 as ms
from test_token_host import refused

pytestmark = pytest.mark.gpu

N, T, D, I, P, K = 4, 45, 256, 136, 2, 3        # ranks, tokens of each, widths, experts of a rank, choices of a token
E = N * P


def moved(s, demand, perm, count):
    """For every matching: (source, destination, first send row, rows, first row at the destination), as the schedule says. On the host: this stands for the links."""
    before = demand.cumsum(-1) - demand
    return [(i, int(perm[k, i]), int(before[i, perm[k, i]] + s["start"][0, k, i]), int(s["length"][0, k, i]), int(s["row"][0, k, i]))
            for k in range(count) for i in range(N) if s["length"][0, k, i] > 0]


def forward(h, r, wn, wr, experts, bits8):
    """One pass over all ranks on this GPU; what the backward pass needs with it."""
    a = ms.rms_norm(h, wn, residual=r, group=64 if bits8 else None, save=True)
    y = a["y"]
    logits = (y.float() @ wr.float().T).contiguous()
    c = ms.route_choose(logits, K, normalise=True)
    d = ms.route_demand(c["experts"][None], E)
    slot = d["slot"][0]
    g = ms.mw_decompose(d["demand"], N * N)
    s = ms.schedule_slots(d["demand"], g.perm, g.dur, g.count, d["counts"])
    assert g.status.item() == 0 and s["status"].item() == 0
    host = {k: v.cpu() for k, v in s.items()}
    moves = moved(host, d["demand"][0].cpu(), g.perm[0].long().cpu(), int(g.count[0]))
    if bits8:
        send, scales = ms.tokens_to_rows(a["q"], slot, scale=a["scale"])
    else:
        send, scales = ms.tokens_to_rows(y, slot), None
    back, ranks = torch.zeros((N, T * K, D), dtype=h.dtype, device="cuda"), []
    for j in range(N):
        R = int(host["rows"][0, j])
        x = torch.zeros((R, D), dtype=send.dtype, device="cuda")
        x_scale = torch.zeros((R, D // 64), device="cuda")
        mine = [m for m in moves if m[1] == j]
        for i, _, first, length, row in mine:
            x[row:row + length] = send[i, first:first + length]
            if bits8:
                x_scale[row:row + length] = scales[i, first:first + length]
        if bits8:
            x = ms.rows_widen(x, x_scale, 64, h.dtype)
        w = [t[j * P:(j + 1) * P].contiguous() for t in experts]
        offsets = s["offsets"][0, j].contiguous()
        out, saved = ms.expert_ffn(x, *w, offsets, save=True)
        for i, _, first, length, row in mine:
            back[i, first:first + length] = out[row:row + length]
        ranks.append((x, w, offsets, saved, mine))
    out = ms.rows_to_tokens(back, slot, K, weights=c["weights"], add=a["sum"])
    return out, dict(a=a, logits=logits, c=c, slot=slot, back=back, ranks=ranks)


def backward(dout, h, r, wn, wr, experts, kept):
    a, c, slot = kept["a"], kept["c"], kept["slot"]
    got = ms.rows_to_tokens_backward(dout, kept["back"], slot, c["weights"])
    dsend, dexperts = torch.zeros((N, T * K, D), dtype=h.dtype, device="cuda"), []
    for x, w, offsets, saved, mine in kept["ranks"]:
        dy = torch.zeros_like(x)
        for i, _, first, length, row in mine:
            dy[row:row + length] = got["drows"][i, first:first + length]
        grads = ms.expert_ffn_backward(dy, x, *w, offsets, saved)
        for i, _, first, length, row in mine:
            dsend[i, first:first + length] = grads["dx"][row:row + length]
        dexperts.append([grads[k] for k in ("dw_gate", "dw_up", "dw_down")])
    dlogits = ms.route_choose_backward(got["dweights"], kept["logits"], c["experts"], normalise=True)
    dy = ms.rows_to_tokens(dsend, slot, K, add=(dlogits @ wr.float()).to(h.dtype))
    dwr = dlogits.flatten(0, 1).T @ a["y"].float().flatten(0, 1)
    n = ms.rms_norm_backward(dy, a["sum"], wn, a["rstd"], dsum=dout)
    return dict(dh=n["dx"], dwn=n["dweight"], dwr=dwr, **{f"dw{q}": torch.cat([d[q] for d in dexperts]) for q in range(3)})


def reference(dout, h, r, wn, wr, experts, chosen, y_sent=None):
    """The layer in 64 bits with the same choices; y_sent: what the experts get instead of y (gradients go to y as if it were y)."""
    leaves = [t.double().requires_grad_() for t in (h, wn, wr, *experts)]
    h64, wn64, wr64, wg, wu, wd = leaves
    s = h64 + r.double()
    y = s * torch.rsqrt((s * s).mean(-1, keepdim=True) + 1e-6) * wn64
    logits = y @ wr64.T
    x = y if y_sent is None else y + (y_sent.double() - y.detach())
    pick = chosen.view(N, T, K).long()
    weights = torch.softmax(torch.gather(logits, 2, pick.clamp_min(0)).masked_fill(pick < 0, -1e30), -1) * (pick >= 0)
    out = s
    for e in range(E):
        f = (torch.nn.functional.silu(x @ wg[e].T) * (x @ wu[e].T)) @ wd[e].T
        out = out + f * (weights * (pick == e)).sum(-1, keepdim=True)
    grads = torch.autograd.grad(out, leaves, dout.double())
    return out.detach(), dict(zip(("dh", "dwn", "dwr", "dw0", "dw1", "dw2"), grads)), logits.detach()


@pytest.mark.parametrize("bits8", [False, True])
def test_a_layer_and_its_gradients(bits8):
    g = torch.Generator("cuda").manual_seed(5)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).half()

    h, r, dout = normal(N, T, D), normal(N, T, D), normal(N, T, D)
    wn, wr = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).half(), normal(E, D, std=D ** -0.5)
    experts = normal(E, I, D, std=D ** -0.5), normal(E, I, D, std=D ** -0.5), normal(E, D, I, std=I ** -0.5)
    out, kept = forward(h, r, wn, wr, experts, bits8)
    grads = backward(dout, h, r, wn, wr, experts, kept)
    sent = ms.rows_widen(kept["a"]["q"], kept["a"]["scale"], 64, torch.float32) if bits8 else None
    want, exact, logits = reference(dout, h, r, wn, wr, experts, kept["c"]["experts"], sent)
    # The choices are those of the logits as the layer has them: y and s are off by half a step of 2^-11 each.
    best = torch.topk(logits, K, -1)
    taken = torch.gather(logits, 2, kept["c"]["experts"].view(N, T, K).long())
    assert ((best.values - taken).abs() <= 2 * 2.0 ** -11 * torch.linalg.norm(wr.double(), dim=-1).max() * D ** 0.5).all()
    # Every tensor on the way is rounded once to 11 bits (relatively 2^-11 of its length): s, y, the experts' h, their y, the sum; backwards drows, dh, da, du, dx, dy and the
    # result. 16 roundings at the most, none of which a later step makes longer relative to what it computes by more than 4 (norms of the products: 2 at most, widths of this size).
    for name, value, ref in [("out", out, want)] + [(k, grads[k], exact[k]) for k in exact]:
        off = (torch.linalg.norm(value.double() - ref) / torch.linalg.norm(ref)).item()
        assert off <= 16 * 4 * 2.0 ** -11, (name, off)


def test_the_checked_library_gives_the_same():
    """The compiled part of the binding calls whichever library is loaded."""
    from paper_2605_26845_b200 import build as cuda_build
    x = torch.randn((50, 264), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    w, l = torch.ones(264, dtype=torch.bfloat16, device="cuda"), torch.randn((50, 24), device="cuda", generator=torch.Generator("cuda").manual_seed(2))

    def run():
        n = ms.rms_norm(x, w, residual=x, group=64, save=True)
        c = ms.route_choose(l, 3, bias=l[0].contiguous())
        slot = ms.route_demand(c["experts"].view(1, 1, -1), 24)["slot"].view(-1)
        rows = ms.tokens_to_rows(n["y"], slot)
        y = ms.rows_to_tokens(rows, slot, 3, weights=c["weights"])
        return [*n.values(), *c.values(), rows, y, *ms.rows_to_tokens_backward(x, rows, slot, c["weights"]).values(),
                *ms.rms_norm_backward(x, n["sum"], w, n["rstd"], dsum=y).values()]

    want = run()
    ms.use_library(cuda_build.build(checked=True))
    try:
        got = run()
        assert ms.debug_index_faults() == 0
    finally:
        ms.use_library(None)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(run(), want))


def test_tensors_without_memory_end_in_an_exception():
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode() as mode:
        x, w = torch.empty((4, 64), device="cuda"), torch.empty(64, device="cuda")
        with pytest.raises(Exception):
            ms.rms_norm(x, w)
    with pytest.raises(Exception):
        ms.rms_norm(x, w, out={"y": x})
    x = torch.zeros((4, 64), device="cuda")
    assert torch.equal(ms.rms_norm(x, x[0])["y"], x)                              # (and the lock is held again)


def test_outputs_of_deterministic_programs_are_filled():
    """Where the program asks for it, memory that a call leaves as it is holds NaN and not whatever was there."""
    x, slot = torch.ones((2, 64), device="cuda"), torch.tensor([1, -1], dtype=torch.int32, device="cuda")
    torch.use_deterministic_algorithms(True)
    try:
        rows = ms.tokens_to_rows(x, slot)
    finally:
        torch.use_deterministic_algorithms(False)
    assert torch.isnan(rows[0]).all() and torch.equal(rows[1], x[0])


def test_calls_from_several_threads():
    import threading
    made = {}

    def work(n):
        with torch.cuda.stream(torch.cuda.Stream()):
            x = torch.full((300, 1032), float(n + 1), device="cuda", dtype=torch.bfloat16)
            w, slot = torch.ones(1032, dtype=torch.bfloat16, device="cuda"), torch.arange(600, dtype=torch.int32, device="cuda")
            for _ in range(50):
                res = ms.rms_norm(x, w, residual=x, save=True, group=128)
                y = ms.rows_to_tokens(ms.tokens_to_rows(res["sum"], slot), slot, 2)
                g = ms.rms_norm_backward(x, res["sum"], w, res["rstd"])["dweight"]
            torch.cuda.current_stream().synchronize()
            made[n] = y, g, res["q"].float()

    threads = [threading.Thread(target=work, args=(n,)) for n in range(6)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for n in range(6):
        y, g, q = made[n]
        assert (y == 4 * (n + 1)).all() and (q == 448).all() and torch.isfinite(g).all() and len(set(g.tolist())) == 1


def test_padding_is_not_sent():
    """Tokens whose logits are all off choose nobody: no demand, no row, and the residual stream goes on as it was."""
    logits = torch.randn((1, 2, 8, 4), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    logits[0, 1, 5:] = -float("inf")
    c = ms.route_choose(logits, 2)
    d = ms.route_demand(c["experts"], 4)
    assert d["demand"][0].sum(-1).tolist() == [16, 10] and (d["status"] == 0).all()
    x = torch.randn((1, 2, 8, 64), device="cuda", generator=torch.Generator("cuda").manual_seed(3)).bfloat16()
    rows = ms.tokens_to_rows(x, d["slot"], out=torch.full((1, 2, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda"))
    assert (rows[0, 1, 10:] == 7).all()
    y = ms.rows_to_tokens(rows, d["slot"], 2, weights=c["weights"], add=x)
    assert torch.equal(y[0, 1, 5:], x[0, 1, 5:])


def test_what_is_refused_on_the_gpu():
    wrong, missing, right = refused(lambda shape, dtype: torch.zeros(shape, dtype=dtype, device="cuda"))
    for call in right:
        call()
    for n, call in enumerate(wrong + missing):
        with pytest.raises(ms.MoeschedError):
            call()
            print("not refused:", n)
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    x, w = torch.zeros((6, 64), dtype=bf, device="cuda"), torch.zeros(64, dtype=bf, device="cuda")
    l, slot, ex = torch.zeros((6, 10), device="cuda"), torch.zeros(12, dtype=i32, device="cuda"), torch.zeros(12, dtype=i32, device="cuda")
    rows, weights, rstd = torch.zeros((12, 64), dtype=bf, device="cuda"), torch.zeros(12, device="cuda"), torch.zeros(6, device="cuda")
    other = torch.zeros((5, 64), dtype=bf, device="cuda")
    host = dict(x=x.cpu(), w=w.cpu(), slot=slot.cpu(), weights=weights.cpu())
    for call in (lambda: ms.rms_norm(x, w, out={"y": other}), lambda: ms.rms_norm(x, w, group=32, out={"q": x}), lambda: ms.rms_norm(x, w, save=True, out={"rstd": weights}),
                 lambda: ms.rms_norm(x, w, out=[x]), lambda: ms.rms_norm(x, w, out={"y": x.t().contiguous().t()}), lambda: ms.rms_norm_backward(x, x, w, rstd, out={"dweight": rstd}),
                 lambda: ms.route_choose(l, 2, out={"experts": ex.view(6, 2)}), lambda: ms.route_choose_backward(weights, l, ex, out=x), lambda: ms.tokens_to_rows(x, slot, out=x),
                 lambda: ms.tokens_to_rows(x, slot, scale=l, out_scale=l), lambda: ms.rows_to_tokens(rows, slot, 2, out=rows), lambda: ms.rows_to_tokens_backward(x, rows, slot, weights, out={"drows": x}),
                 lambda: ms.rows_to_tokens(rows, slot, 2, out=x.float()), lambda: ms.rms_norm(x, host["w"]), lambda: ms.rms_norm(host["x"], w), lambda: ms.tokens_to_rows(x, host["slot"]),
                 lambda: ms.rows_to_tokens(rows, slot, 2, weights=host["weights"]), lambda: ms.rms_norm(x, w, out={"y": host["x"]}),
                 lambda: ms.rms_norm(torch.zeros(6 * 64 + 1, dtype=bf, device="cuda")[1:].view(6, 64), w)):       # (the last one is not on 16 bytes)
        with pytest.raises(ms.MoeschedError):
            call()
    assert torch.equal(ms.rms_norm(x, w, out={})["y"], x)
