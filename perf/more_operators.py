"""Timed work of the operators between a layer's tokens and the send buffers: the norm before the router, the router's choice, the
tokens' way into the rows that are sent, by expert, and back.

listed() holds the named cases, draw() makes further ones of the same ranges. Ops:
  norm    root-mean-square norm of tokens, with the residual's addition, an output in 8 bits with scales (group > 0), gradients (train)
  choose  the k experts of every token and their weights from the router's logits; train=True adds the logits' gradient
  send    tokens to rows by expert; train=True adds the tokens' gradient
  send8   the same in 8 bits with scales, and the rows widened again where they arrive
  back    rows to tokens, weights applied, the residual added where add=True; train=True adds the gradients of rows and weights

run() computes the plain form in 32 bits (64 for the scores that a choice is made by); with own = True it calls the framework.
"""
import math

import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def _norm(T, D, dtype, residual, group, train, name=None):
    c = dict(op="norm", T=T, D=D, dtype=dtype, residual=residual, group=group, train=train)
    return dict(c, name=name) if name else c


def _choose(T, E, k, dtype, score, bias, normalise, train, name=None):
    c = dict(op="choose", T=T, E=E, k=k, dtype=dtype, score=score, bias=bias, normalise=normalise, train=train)
    return dict(c, name=name) if name else c


def _send(T, D, k, dtype, train, name=None):
    c = dict(op="send", T=T, D=D, k=k, E=64, dtype=dtype, train=train)
    return dict(c, name=name) if name else c


def _send8(T, D, k, dtype, group, name=None):
    c = dict(op="send8", T=T, D=D, k=k, E=64, dtype=dtype, group=group)
    return dict(c, name=name) if name else c


def _back(T, D, k, dtype, add, train, name=None):
    c = dict(op="back", T=T, D=D, k=k, E=64, dtype=dtype, add=add, train=train)
    return dict(c, name=name) if name else c


def listed():
    return [
        # decoding, one token: nothing but latency
        _norm(1, 7168, "bf16", True, 128, False, name="norm_one"),
        # the tokens of a rank's prefill, sent in 8 bits
        _norm(16384, 7168, "bf16", True, 128, False, name="norm_prefill_16384"),
        # a training step, the residual's gradient comes in from behind
        _norm(8191, 4096, "bf16", True, 0, True, name="norm_train_8191"),
        # decoding: a small batch, choices by the logistic function with a bias that balances the experts
        _choose(16, 256, 8, "fp32", "sigmoid", True, True, False, name="choose_16"),
        # a training step of a layer with 256 experts
        _choose(16384, 256, 8, "fp32", "softmax", False, True, True, name="choose_train_16384"),
        # decoding: the rows of a small batch
        _send(16, 7168, 8, "bf16", False, name="send_16"),
        # a training step, and the gradient on its way back
        _send(8191, 4096, 8, "bf16", True, name="send_train_8191"),
        # decoding in 8 bits, ragged
        _send8(61, 7168, 8, "bf16", 128, name="send8_61"),
        # prefill in 8 bits
        _send8(16384, 7168, 8, "bf16", 128, name="send8_16384"),
        # decoding: back to the residual stream
        _back(16, 7168, 8, "bf16", True, False, name="back_16"),
        # a training step of a small layer, odd sizes
        _back(777, 1000, 3, "fp16", False, True, name="back_train_777"),
        # a training step of a large one
        _back(8191, 4096, 8, "bf16", True, True, name="back_train_8191"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "norm", "choose", "choose", "send", "send8", "back", "back"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    D, k, train = 8 * _log(rng, 16, 896), rng.choice((1, 2, 3, 4, 6, 8)), rng.random() < 0.5
    T = _log(rng, 1, min(16384, 100_000_000 // D))
    if op == "norm":
        return _norm(T, D, dtype, rng.random() < 0.7, 0 if train else rng.choice((0, 32, 64, 128)), train)
    if op == "choose":
        E = rng.choice((8, 16, 60, 64, 128, 160, 256, 512, 1024))
        return _choose(_log(rng, 1, min(16384, 8_000_000 // E)), E, k, rng.choice(("fp32", "fp32", "bf16")), rng.choice(("softmax", "sigmoid")),
                       rng.random() < 0.5, rng.random() < 0.5, train)
    T = max(1, min(T, 400_000_000 // (k * D)))
    if op == "send":
        return _send(T, D, k, dtype, train)
    if op == "send8":
        return _send8(T, D, k, dtype, rng.choice((32, 64, 128)))
    return _back(T, D, k, dtype, rng.random() < 0.5, train)


# ---- inputs --------------------------------------------------------------------------------------------

def _slots(T, k, E, g):
    """Row of every choice among the choices sorted by expert, -1 for one in a hundred that is not sent. Experts are of uneven popularity."""
    popular = torch.rand((E,), generator=g, device=DEVICE).argsort().add(1).double().pow(-0.7).log()
    noise = -torch.log(-torch.log(torch.rand((T, E), generator=g, device=DEVICE, dtype=torch.float64).clamp_(1e-12, 1 - 1e-12)))
    expert = torch.topk(popular + noise, k, dim=-1).indices.reshape(-1)      # k different ones
    expert[torch.rand((T * k,), generator=g, device=DEVICE) > 0.99] = E
    order = torch.sort(expert, stable=True).indices
    slot = torch.empty(T * k, dtype=torch.int32, device=DEVICE)
    slot[order] = torch.arange(T * k, dtype=torch.int32, device=DEVICE)
    slot[expert == E] = -1
    return slot


def prepare(case, seed):
    g = torch.Generator(DEVICE)
    g.manual_seed(seed)
    op, s, dtype = case["op"], {"case": case}, TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32).mul_(std).to(dtype)

    T = case["T"]
    if op == "choose":
        E, k = case["E"], case["k"]
        logits = torch.randn((T, E), generator=g, device=DEVICE) * 1.5
        padded = torch.rand((T, 1), generator=g, device=DEVICE) > 0.99      # tokens that fill up a batch choose nobody
        s["logits"] = torch.where(padded, -math.inf, logits).to(dtype)
        s["bias"] = torch.randn((E,), generator=g, device=DEVICE) * 0.05 if case["bias"] else None
        s["dweights"] = torch.randn((T * k,), generator=g, device=DEVICE)
        return s
    D = case["D"]
    if op == "norm":
        loud = torch.where(torch.rand((D,), generator=g, device=DEVICE) < 0.005, 20.0, 1.0)      # a few channels are much larger
        s["x"] = (normal(T, D).float() * loud).to(dtype)
        s["weight"] = (1 + 0.1 * torch.randn((D,), generator=g, device=DEVICE)).to(dtype)
        s["residual"] = normal(T, D, std=2.0) if case["residual"] else None
        if case["train"]:
            s["dy"], s["dsum"] = normal(T, D), normal(T, D) if case["residual"] else None
        return s
    k = case["k"]
    s["slot"] = _slots(T, k, case["E"], g)
    if op == "send8":
        s["x"] = (normal(T, D).float() * 60).clamp_(-448, 448).to(torch.float8_e4m3fn)
        P = -(-D // case["group"])
        s["scale"] = torch.rand((T, P), generator=g, device=DEVICE) * 0.02 + 0.002
        s["rows"] = torch.zeros((T * k, D), dtype=torch.float8_e4m3fn, device=DEVICE)       # the send buffer
        s["row_scale"] = torch.zeros((T * k, P), device=DEVICE)
    elif op == "send":
        s["x"] = normal(T, D)
        s["rows"] = torch.zeros((T * k, D), dtype=dtype, device=DEVICE)
        if case["train"]:
            s["drows"] = normal(T * k, D)
    else:
        s["rows"] = normal(T * k, D)
        s["weights"] = torch.rand((T * k,), generator=g, device=DEVICE)
        s["add"] = normal(T, D) if case["add"] else None
        if case["train"]:
            s["dy"] = normal(T, D)
            s["drows"] = torch.zeros((T * k, D), dtype=dtype, device=DEVICE)
    return s


# ---- one pass ------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"norm": _plain_norm, "choose": _plain_choose, "send": _plain_send, "send8": _plain_send8, "back": _plain_back}[case["op"]](s, case)


def _run_own(s, case):
    import paper_2605_26845_b200 as ms

    op = case["op"]
    if op == "norm":
        r = ms.rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], group=case["group"] or None, save=case["train"])
        out = {n: r[n] for n in ("y", "sum", "q", "scale") if n in r}
        if case["train"]:
            out.update(ms.rms_norm_backward(s["dy"], r.get("sum", s["x"]), s["weight"], r["rstd"], dsum=s["dsum"]))
        return out
    if op == "choose":
        how = dict(score=case["score"], bias=s["bias"], normalise=case["normalise"], factor=2.5)
        out = ms.route_choose(s["logits"], case["k"], **how)
        if case["train"]:
            del how["bias"]
            out["dlogits"] = ms.route_choose_backward(s["dweights"], s["logits"], out["experts"], **how)
        return out
    if op == "send":
        out = {"rows": ms.tokens_to_rows(s["x"], s["slot"], out=s["rows"])}
        if case["train"]:
            out["dx"] = ms.rows_to_tokens(s["drows"], s["slot"], case["k"])
        return out
    if op == "send8":
        rows, scale = ms.tokens_to_rows(s["x"], s["slot"], scale=s["scale"], out=s["rows"], out_scale=s["row_scale"])
        return {"rows": rows, "scale": scale, "wide": ms.rows_widen(rows, scale, case["group"], TYPES[case["dtype"]])}
    out = {"y": ms.rows_to_tokens(s["rows"], s["slot"], case["k"], weights=s["weights"], add=s["add"])}
    if case["train"]:
        out.update(ms.rows_to_tokens_backward(s["dy"], s["rows"], s["slot"], s["weights"], out={"drows": s["drows"]}))
    return out


def _plain_norm(s, case):
    x, w, dtype = s["x"].float(), s["weight"].float(), s["x"].dtype
    out = {}
    if case["residual"]:
        out["sum"] = (x + s["residual"].float()).to(dtype)          # the residual stream, as it is kept
        x = out["sum"].float()
    c = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    y = x * c * w
    out["y"] = y.to(dtype)
    if case["group"]:
        G, D = case["group"], case["D"]
        P = -(-D // G)
        parts = torch.nn.functional.pad(y, (0, P * G - D)).view(case["T"], P, G)
        out["scale"] = (parts.abs().amax(-1) / 448).clamp_min(2.0 ** -126)
        q = (parts / out["scale"][..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        out["q"] = q.view(case["T"], P * G)[:, :D].contiguous()
    if case["train"]:
        dy = s["dy"].float()
        g = dy * w
        dx = c * (g - x * (c * c * (g * x).mean(-1, keepdim=True)))
        if case["residual"]:
            dx = dx + s["dsum"].float()
        out["dx"], out["dweight"] = dx.to(dtype), (dy * x * c).sum(0).to(dtype)
    return out


def _plain_scores(logits, kind):
    """Scores of the experts; 0 throughout where none may be chosen."""
    if kind == "sigmoid":
        return torch.sigmoid(logits)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
    return p / p.sum(-1, keepdim=True).clamp_min(torch.finfo(p.dtype).tiny)


def _plain_choose(s, case):
    l, k, factor = s["logits"].float(), case["k"], 2.5
    wide = _plain_scores(l.double(), case["score"]) + s["bias"].double() if case["bias"] else l.double()
    wide = torch.where(l == -math.inf, -math.inf, wide)
    best = torch.sort(wide, dim=-1, descending=True, stable=True)
    chosen, there = best.indices[:, :k], best.values[:, :k] > -math.inf
    p = _plain_scores(l, case["score"])
    score = torch.gather(p, 1, chosen) * there
    total = score.sum(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).tiny)
    weights = factor * (score / total if case["normalise"] else score)
    out = {"experts": torch.where(there, chosen, -1).int().reshape(-1), "weights": weights.reshape(-1)}
    if case["train"]:
        dw = factor * s["dweights"].view(-1, k) * there
        if case["normalise"]:
            dscore = (dw - (dw * score / total).sum(-1, keepdim=True)) / total * there
        else:
            dscore = dw
        d = torch.zeros_like(p).scatter_add_(1, chosen, dscore)     # (a token's experts are different ones)
        d = p * (1 - p) * d if case["score"] == "sigmoid" else p * (d - (d * p).sum(-1, keepdim=True))
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _plain_rows(x, slot, k):
    """The row of token t at the places of its choices; rows that nobody takes are 0."""
    S = slot.numel()
    rows = torch.zeros((S + 1, x.shape[1]), dtype=x.dtype, device=x.device)
    token = torch.div(torch.arange(S, device=slot.device), k, rounding_mode="floor")
    rows[torch.where(slot < 0, S, slot).long()] = x[token]
    return rows[:S]


def _plain_picked(rows, slot, k):
    """[T, k, D] in 32 bits: the rows of every token's choices, 0 for those that were not sent."""
    picked = rows[slot.clamp_min(0).long()].float() * (slot >= 0)[:, None]
    return picked.view(-1, k, rows.shape[1])


def _plain_send(s, case):
    out = {"rows": _plain_rows(s["x"].float(), s["slot"], case["k"]).to(s["x"].dtype)}
    if case["train"]:
        out["dx"] = _plain_picked(s["drows"], s["slot"], case["k"]).sum(1).to(s["x"].dtype)
    return out


def _plain_send8(s, case):
    rows = _plain_rows(s["x"].float(), s["slot"], case["k"])
    scale = _plain_rows(s["scale"], s["slot"], case["k"])
    wide = rows * scale.repeat_interleave(case["group"], 1)[:, : case["D"]]
    return {"rows": rows.to(torch.float8_e4m3fn), "scale": scale, "wide": wide.to(TYPES[case["dtype"]])}


def _plain_back(s, case):
    k, dtype = case["k"], s["rows"].dtype
    picked = _plain_picked(s["rows"], s["slot"], k)
    y = (picked * s["weights"].view(-1, k, 1)).sum(1)
    if case["add"]:
        y = y + s["add"].float()
    out = {"y": y.to(dtype)}
    if case["train"]:
        dy = s["dy"].float()
        out["dweights"] = (picked * dy[:, None]).sum(-1).reshape(-1)
        S = case["T"] * k
        drows = torch.zeros((S + 1, case["D"]), device=dy.device)
        drows[torch.where(s["slot"] < 0, S, s["slot"]).long()] = (dy[:, None] * s["weights"].view(-1, k, 1)).view(S, -1)
        out["drows"] = drows[:S].to(dtype)
    return out


# ---- what a pass cannot do without, and its result in 64 bits -------------------------------------------

def work(case):
    op, T = case["op"], case["T"]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if op == "choose":
        E, k = case["E"], case["k"]
        moved = T * E * size + 8 * T * k
        return {"bytes": moved + (T * E * size + 4 * T * k if case["train"] else 0), "flops": 5 * T * E * (2 if case["train"] else 1)}
    D = case["D"]
    if op == "norm":
        tensors = (4 if case["residual"] else 2) + ((3 if case["residual"] else 2) if case["train"] else 0)
        q = T * (D + 4 * -(-D // case["group"])) if case["group"] else 0
        return {"bytes": tensors * T * D * size + q + D * size, "flops": (20 if case["train"] else 6) * T * D}
    S = case["T"] * case["k"]
    sent = S * 99 // 100
    if op == "send":
        one = T * D * size + sent * D * size
        return {"bytes": 4 * S + one * (2 if case["train"] else 1), "flops": sent * D if case["train"] else 0}
    if op == "send8":
        P = -(-D // case["group"])
        return {"bytes": 4 * S + (T + sent) * (D + 4 * P) + sent * D * size, "flops": sent * D}
    moved = sent * D * size + T * D * size * (2 if case["add"] else 1) + 8 * S
    if case["train"]:
        moved += sent * D * size + T * D * size + 4 * S
    return {"bytes": moved, "flops": (5 if case["train"] else 2) * sent * D}


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    T = case["T"]
    if op == "norm":
        h, w = s["x"].double(), s["weight"].double()
        out = {}
        if case["residual"]:
            out["sum"] = h + s["residual"].double()
            h = out["sum"].to(s["x"].dtype).double()
        c = 1 / torch.sqrt(torch.einsum("td,td->t", h, h) / case["D"] + EPS)
        out["y"] = torch.einsum("td,t,d->td", h, c, w)
        if case["group"]:
            edges = range(0, case["D"], case["group"])
            out["scale"] = torch.stack([out["y"][:, e : e + case["group"]].abs().max(-1).values / 448 for e in edges], -1).clamp(min=2.0 ** -126)
            out["q"] = out["y"] / out["scale"].repeat_interleave(case["group"], -1)[:, : case["D"]]
        if case["train"]:
            # h -> h / |h|: the part of the gradient along h falls away, but for eps
            dy = s["dy"].double()
            along = torch.einsum("td,d,td->t", dy, w, h) * c ** 3 / case["D"]
            out["dx"] = dy * w * c[:, None] - h * along[:, None] + (s["dsum"].double() if case["residual"] else 0)
            out["dweight"] = torch.einsum("td,td,t->d", dy, h, c)
        return out
    if op == "choose":
        l, k = s["logits"].double(), case["k"]
        if case["score"] == "softmax":
            score = torch.nan_to_num(torch.softmax(l, -1), nan=0.0)
        else:
            score = 1 / (1 + torch.exp(-l))
        l = l.requires_grad_() if case["train"] else l
        rank = score + s["bias"].double() if case["bias"] else s["logits"].double()
        rank = rank.masked_fill(s["logits"] == -math.inf, -math.inf)
        chosen = torch.argsort(rank, dim=-1, descending=True, stable=True)[:, :k]
        padded = (s["logits"] == -math.inf).all(-1)
        with torch.enable_grad():
            live = l[~padded]
            p = torch.softmax(live, -1) if case["score"] == "softmax" else torch.special.expit(live)
            p = torch.gather(p, 1, chosen[~padded])
            w = 2.5 * (p / p.sum(-1, keepdim=True) if case["normalise"] else p)
        out = {"experts": None, "weights": torch.zeros((T, k), dtype=torch.float64, device=DEVICE)}
        out["weights"][~padded] = w.detach()
        out["weights"] = out["weights"].view(-1)
        if case["train"]:
            (out["dlogits"],) = torch.autograd.grad(w, l, s["dweights"].double().view(T, k)[~padded])
        return out
    D, k, slot = case["D"], case["k"], s["slot"].long()
    sent = torch.nonzero(slot >= 0)[:, 0]

    def placed(values):
        out = torch.zeros((T * k, values.shape[1]), dtype=torch.float64, device=DEVICE)
        out.index_copy_(0, slot[sent], values.double())
        return out

    if op == "send":
        out = {"rows": placed(s["x"][sent // k])}
        if case["train"]:
            out["dx"] = torch.zeros((T, D), dtype=torch.float64, device=DEVICE).index_add_(0, sent // k, s["drows"][slot[sent]].double())
        return out
    if op == "send8":
        rows, scale = placed(s["x"].to(torch.float32)[sent // k]), placed(s["scale"][sent // k])
        factor = scale[:, torch.arange(D, device=DEVICE) // case["group"]]
        return {"rows": rows, "scale": scale, "wide": rows * factor}
    w = s["weights"].double()[sent]
    y = s["add"].double() if case["add"] else torch.zeros((T, D), dtype=torch.float64, device=DEVICE)
    y = y.index_add(0, sent // k, s["rows"][slot[sent]].double() * w[:, None])
    out = {"y": y}
    if case["train"]:
        dy = s["dy"].double()[sent // k]
        out["drows"] = placed(dy * w[:, None])
        out["dweights"] = torch.zeros(T * k, dtype=torch.float64, device=DEVICE)
        out["dweights"][sent] = torch.einsum("sd,sd->s", dy, s["rows"][slot[sent]].double())
    return out
