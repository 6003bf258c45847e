"""Timed work of the operators around a schedule: what is sent, where it lands, and the experts that compute on it.

listed() holds the named cases, draw() makes further ones of the same ranges. Ops:
  route   router's choices of a batch of all-to-alls -> demand matrices, counts per expert, slots of the send buffers
  slots   demand and schedule -> first token, length and receiver's row of every transfer, offsets of the expert batches
  ffn     gated feed-forward block of the experts of a rank on rows grouped by expert; train=True adds the backward pass
  matvec4 product of a few rows with the experts' 4-bit weights, plain or gated

run() computes the plain form in 32 bits; with own = True it calls the framework.
"""
import math

import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _route(N, B, S, per_rank, name=None):
    c = dict(op="route", N=N, B=B, S=S, per_rank=per_rank)
    return dict(c, name=name) if name else c


def _slots(N, B, K, per_rank, rounds, name=None):
    c = dict(op="slots", N=N, B=B, K=K, per_rank=per_rank, rounds=rounds)
    return dict(c, name=name) if name else c


def _ffn(E, D, I, R, matchings, train, dtype, act="silu", name=None):
    c = dict(op="ffn", E=E, D=D, I=I, R=R, matchings=matchings, train=train, dtype=dtype, act=act)
    return dict(c, name=name) if name else c


def _matvec4(E, K, N, R, group, gated, dtype, name=None):
    c = dict(op="matvec4", E=E, K=K, N=N, R=R, group=group, gated=gated, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one layer of eight ranks, two choices for each of 4096 tokens: nothing but latency
        _route(8, 1, 4096 * 2, 1, name="route_n8_b1"),
        # the layers of a step on 64 ranks, eight choices for each of 16384 tokens, 256 experts
        _route(64, 16, 16384 * 8, 4, name="route_n64_b16"),
        # greedy schedules of a few layers on 16 ranks
        _slots(16, 24, 16, 4, 1, name="slots_n16_b24"),
        # greedy schedules of many layers and steps on 64 ranks, complete
        _slots(64, 1024, 64, 4, 1, name="slots_n64_b1024"),
        # a Birkhoff schedule: the pairs come back in pieces, many matchings
        _slots(128, 4, 2304, 4, 18, name="slots_n128_b4_pieces"),
        # decoding: the handful of tokens of one small matching on a rank with four experts
        _ffn(4, 7168, 2048, 16, 1, False, "bf16", name="ffn_decode_16"),
        # one matching's batch, ragged over the experts
        _ffn(4, 7168, 2048, 2051, 1, False, "bf16", name="ffn_matching_2051"),
        # everything a rank receives in one all-to-all, in the order in which five matchings brought it
        _ffn(4, 7168, 2048, 32768, 5, False, "bf16", name="ffn_prefill_32768"),
        # a training step of a small layer
        _ffn(8, 1000, 704, 777, 2, True, "fp16", "gelu", name="ffn_train_777"),
        # a training step of a rank with eight experts
        _ffn(8, 4096, 2048, 16384, 1, True, "bf16", name="ffn_train_16384"),
        # one token at one expert in 4 bits: gate and up projection
        _matvec4(4, 7168, 2048, 1, 128, True, "bf16", name="matvec4_one_gated"),
        # a decoding batch spread over 32 experts: down projection
        _matvec4(32, 2048, 7168, 61, 64, False, "fp16", name="matvec4_61_down"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("route", "slots", "ffn", "ffn", "train", "matvec4"))
    dtype = rng.choice(("bf16", "fp16"))
    if op == "route":
        N = _log(rng, 2, 128)
        per_rank = rng.choice((1, 2, 3, 4, 8))
        S = _log(rng, 100, 131072)
        return _route(N, _log(rng, 1, max(1, min(64, 100_000_000 // (N * S)))), S, per_rank)
    if op == "slots":
        N = _log(rng, 2, 128)
        rounds = rng.choice((1, 1, 3, 9))
        K = N * rounds - rng.randrange(N)
        return _slots(N, _log(rng, 1, max(1, min(1024, 3_000_000 // (N * K)))), K, rng.choice((1, 2, 3, 4)), rounds)
    if op == "matvec4":
        group = rng.choice((32, 64, 128))
        K = group * _log(rng, max(1, 256 // group), 7168 // group)
        return _matvec4(rng.choice((1, 2, 4, 8, 32)), K, 8 * _log(rng, 32, 896), _log(rng, 1, 96), group, rng.random() < 0.5, dtype)
    E = rng.choice((1, 2, 3, 4, 8))
    D, I = 8 * _log(rng, 32, 896), 8 * _log(rng, 32, 256)
    return _ffn(E, D, I, _log(rng, 1, min(16384, 120_000_000_000 // (D * I))), rng.choice((1, 1, 2, 5)), op == "train", dtype, rng.choice(("silu", "silu", "gelu")))


# ---- inputs --------------------------------------------------------------------------------------------

def _generators(seed):
    g = torch.Generator(DEVICE)
    g.manual_seed(seed)
    h = torch.Generator("cpu")
    h.manual_seed(seed)
    return g, h


def _popularity(shape, g):
    """Zipf weights over the last dimension, in an order of its own for every row."""
    n = shape[-1]
    order = torch.rand(shape, generator=g, device=g.device).argsort(dim=-1)
    return (order + 1).double() ** -1.0


def _lengths(groups, R, h):
    """Rows of every group: Zipf shares of R, some groups empty, in random order."""
    share = _popularity((groups,), h)
    share = torch.where(torch.rand(groups, generator=h) < 0.1, torch.zeros_like(share), share)
    share[int(torch.randint(groups, (1,), generator=h))] += 0.1
    edge = (share.cumsum(0) / share.sum() * R).round().long()
    edge[-1] = R
    return torch.diff(edge, prepend=torch.zeros(1, dtype=torch.long))


def prepare(case, seed):
    g, h = _generators(seed)
    op, s = case["op"], {"case": case}

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32).mul_(std).to(TYPES[case["dtype"]])

    if op == "route":
        N, B, S = case["N"], case["B"], case["S"]
        E = N * case["per_rank"]
        cum = _popularity((B, 1, E), g).cumsum(-1)
        cum = (cum / cum[..., -1:]).float().contiguous()
        s["experts"] = torch.empty((B, N, S), dtype=torch.int32, device=DEVICE)
        for b in range(B):
            at = torch.rand((N, S), generator=g, device=DEVICE)
            s["experts"][b] = torch.searchsorted(cum[b, 0], at).clamp_(max=E - 1)
            s["experts"][b][at > 0.99] = -1         # tokens that were dropped, and padding
        s["E"] = E
    elif op == "slots":
        N, B, K, P, rounds = (case[k] for k in ("N", "B", "K", "per_rank", "rounds"))
        share = _popularity((B, 1, N * P), g)
        s["counts"] = (torch.rand((B, N, N * P), generator=g, device=DEVICE) * share * 2000).int()
        s["demand"] = s["counts"].view(B, N, N, P).sum(-1, dtype=torch.int32)
        # every round holds the N rotations of the ranks (relabelled, in random order): all pairs once
        label = torch.rand((B, N), generator=g, device=DEVICE).argsort(-1)
        back = label.argsort(-1)
        shift = torch.rand((B, rounds, N), generator=g, device=DEVICE).argsort(-1).view(B, rounds * N)[:, :K]
        to = (label[:, None, :] + shift[:, :, None]) % N
        perm = torch.gather(back[:, None, :].expand(B, K, N), 2, to)
        s["perm"] = perm.to(torch.uint8)
        pair = torch.gather(s["demand"][:, None].expand(B, K, N, N), 3, perm[..., None])[..., 0] if B * K * N * N < 1 << 31 else None
        if pair is None:
            pair = torch.stack([torch.gather(s["demand"][b], 1, perm[b].T).T for b in range(B)])
        heaviest = pair.amax(-1)
        s["dur"] = torch.div(heaviest + rounds - 1, rounds, rounding_mode="floor").int().clamp_(min=1)
        count = torch.randint(max(1, K - K // 8), K + 1, (B,), generator=g, device=DEVICE)
        s["count"] = count.int()
    elif op == "ffn":
        E, D, I, R = (case[k] for k in ("E", "D", "I", "R"))
        lengths = _lengths(E * case["matchings"], R, h)
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.long), lengths.cumsum(0)]).int().to(DEVICE)
        s["most"] = int(lengths.view(-1, E).sum(0).max())
        s["x"] = normal(R, D)
        s["w_gate"], s["w_up"], s["w_down"] = normal(E, I, D, std=D ** -0.5), normal(E, I, D, std=D ** -0.5), normal(E, D, I, std=I ** -0.5)
        if case["train"]:
            s["dy"] = normal(R, D)
    else:
        E, K, N, R, G = (case[k] for k in ("E", "K", "N", "R", "group"))
        lengths = _lengths(E, R, h)
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.long), lengths.cumsum(0)]).int().to(DEVICE)
        s["most"] = int(lengths.max())
        s["x"] = normal(R, K)
        for part in ("w", "up")[: 2 if case["gated"] else 1]:
            s[part] = torch.randint(0, 256, (E, N, K // 2), generator=g, device=DEVICE, dtype=torch.uint8)
            s[part + "_scale"] = (torch.rand((E, N, K // G), generator=g, device=DEVICE) * 0.03 + 0.005).to(TYPES[case["dtype"]])
    return s


# ---- one pass ------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"route": _plain_route, "slots": _plain_slots, "ffn": _plain_ffn, "matvec4": _plain_matvec4}[case["op"]](s, case)


def _run_own(s, case):
    import paper_2605_26845_b200 as ms

    op = case["op"]
    if op == "route":
        r = ms.route_demand(s["experts"], s["E"])
        return {k: r[k] for k in ("demand", "counts", "slot")}
    if op == "slots":
        r = ms.schedule_slots(s["demand"], s["perm"], s["dur"], s["count"], s["counts"])
        return {k: r[k] for k in ("start", "length", "row", "rows", "offsets")}
    if op == "matvec4":
        return ms.expert_matvec4(s["x"], s["w"], s["w_scale"], s["offsets"], s.get("up"), s.get("up_scale"))
    weights = s["w_gate"], s["w_up"], s["w_down"]
    if not case["train"]:
        return ms.expert_ffn(s["x"], *weights, s["offsets"], act=case["act"])
    y, saved = ms.expert_ffn(s["x"], *weights, s["offsets"], act=case["act"], save=True)
    return {"y": y, **ms.expert_ffn_backward(s["dy"], s["x"], *weights, s["offsets"], saved, act=case["act"])}


def _plain_route(s, case):
    N, P, E = case["N"], case["per_rank"], s["E"]
    e = s["experts"].long()
    B, _, S = e.shape
    key = torch.where(e < 0, E, e)
    order = torch.sort(key, dim=-1, stable=True).indices
    slot = torch.empty_like(s["experts"])
    slot.scatter_(2, order, torch.arange(S, dtype=torch.int32, device=e.device).expand(B, N, S))
    slot = torch.where(e < 0, -1, slot)
    counts = torch.zeros((B, N, E + 1), dtype=torch.int32, device=e.device)
    counts.scatter_add_(2, key, torch.ones((), dtype=torch.int32, device=e.device).expand(B, N, S))
    counts = counts[..., :E].contiguous()
    return {"demand": counts.view(B, N, N, P).sum(-1, dtype=torch.int32), "counts": counts, "slot": slot}


def _plain_slots(s, case):
    N, P, K = case["N"], case["per_rank"], case["K"]
    demand, B = s["demand"].long(), case["B"]
    used = torch.arange(K, device=demand.device)[None, :, None] < s["count"].long()[:, None, None]
    to = s["perm"].long()                                                   # [B, K, N]: destination of source i
    dur = (s["dur"].long()[:, :, None] * used).expand(B, K, N)
    # tokens of the pair that earlier matchings could carry: sums of the durations within equal destinations
    dest, order = torch.sort(to, dim=1, stable=True)
    run_ = torch.gather(dur, 1, order)
    before = run_.cumsum(1) - run_
    first = torch.searchsorted(dest.transpose(1, 2).contiguous(), dest.transpose(1, 2).contiguous()).transpose(1, 2)
    earlier = torch.zeros_like(before).scatter_(1, order, before - torch.gather(before, 1, first))
    pair = torch.gather(demand, 2, to.transpose(1, 2)).transpose(1, 2)      # demand of (i, to[k, i])
    start = torch.minimum(pair, earlier) * used
    length = torch.minimum(pair - start, dur) * used
    arrived = torch.zeros_like(length).scatter_(2, to, length)              # by receiver
    begins = arrived.cumsum(1) - arrived
    row = torch.gather(begins, 2, to) * used
    rows = arrived.sum(1)
    # expert batches of receiver j in matching k: the pair's tokens lie by expert
    source = torch.zeros_like(to).scatter_(2, to, torch.arange(N, device=to.device).expand(B, K, N))
    ahead = s["counts"].long().view(B, N, N, P)
    ahead = (ahead.cumsum(-1) - ahead)[torch.arange(B, device=to.device)[:, None, None], source,
                                       torch.arange(N, device=to.device)]      # [B, K, N (receiver), P]
    skipped = torch.gather(start, 2, source)[..., None]
    inside = torch.minimum((ahead - skipped).clamp_(min=0), arrived[..., None])
    offsets = (begins[..., None] + inside).permute(0, 2, 1, 3).reshape(B, N, K * P)
    offsets = torch.cat([offsets, rows[..., None]], -1)
    return {k: v.int() for k, v in (("start", start), ("length", length), ("row", row), ("rows", rows), ("offsets", offsets))}


def _act(a, kind):
    return a * torch.sigmoid(a) if kind == "silu" else 0.5 * a * (1 + torch.erf(a * 0.5 ** 0.5))


def _act_slope(a, kind):
    if kind == "silu":
        z = torch.sigmoid(a)
        return z * (1 + a * (1 - z))
    return 0.5 * (1 + torch.erf(a * 0.5 ** 0.5)) + a * torch.exp(-0.5 * a * a) * (2 * math.pi) ** -0.5


def _by_expert(offsets, R, E):
    """Expert of every row, and its place among the expert's rows."""
    group = torch.searchsorted(offsets, torch.arange(R, device=offsets.device, dtype=torch.int32), right=True) - 1
    expert = group % E
    mine = expert[:, None] == torch.arange(E, device=offsets.device)
    return expert, torch.gather(mine.cumsum(0), 1, expert[:, None])[:, 0] - 1


def _plain_ffn(s, case):
    E, R, kind, x = case["E"], case["R"], case["act"], s["x"]
    at = _by_expert(s["offsets"], R, E)
    gate, up, down = s["w_gate"].float(), s["w_up"].float(), s["w_down"].float()

    def padded(rows):
        p = torch.zeros((E, s["most"], rows.shape[1]), dtype=torch.float32, device=rows.device)
        p[at] = rows.float()
        return p

    xp = padded(x)
    a, u = xp @ gate.mT, xp @ up.mT
    h = _act(a, kind) * u
    y = (h @ down.mT)[at].to(x.dtype)
    if not case["train"]:
        return y
    dyp = padded(s["dy"])
    dh = dyp @ down
    da, du = dh * u * _act_slope(a, kind), dh * _act(a, kind)
    out = {"y": y, "dx": (da @ gate + du @ up)[at], "dw_gate": da.mT @ xp, "dw_up": du.mT @ xp, "dw_down": dyp.mT @ h}
    return {k: v.to(x.dtype) for k, v in out.items()}


def _plain_matvec4(s, case):
    E, R, G, x = case["E"], case["R"], case["group"], s["x"]
    at = _by_expert(s["offsets"], R, E)
    xp = torch.zeros((E, s["most"], case["K"]), dtype=torch.float32, device=x.device)
    xp[at] = x.float()

    def product(part):
        q = s[part]
        w = torch.stack([q & 15, q >> 4], -1).float() - 8                   # low half first
        w = w.view(E, case["N"], -1, G) * s[part + "_scale"].float()[..., None]
        return xp @ w.view(E, case["N"], -1).mT

    y = product("w")
    if case["gated"]:
        y = _act(y, "silu") * product("up")
    return y[at].to(x.dtype)


# ---- what a pass cannot do without, and its result in 64 bits -------------------------------------------

def work(case):
    op = case["op"]
    if op == "route":
        B, N, S = case["B"], case["N"], case["S"]
        return {"bytes": 4 * (2 * B * N * S + B * N * N * (1 + case["per_rank"])), "flops": 0}
    if op == "slots":
        B, N, K, P = case["B"], case["N"], case["K"], case["per_rank"]
        read = 4 * B * N * N * (1 + P) + B * K * (N + 4)
        return {"bytes": read + 4 * (3 * B * K * N + B * N * (K * P + 2)), "flops": 0}
    busy = min(case["E"], case["R"])
    if op == "matvec4":
        parts = 2 if case["gated"] else 1
        weights = parts * busy * case["N"] * (case["K"] // 2 + 2 * case["K"] // case["group"])
        return {"bytes": weights + 2 * case["R"] * (case["K"] + case["N"]), "flops": 2 * parts * case["R"] * case["K"] * case["N"]}
    D, I, R, E = (case[k] for k in ("D", "I", "R", "E"))
    if case["train"]:
        return {"bytes": 2 * (4 * R * D + 6 * E * D * I), "flops": 18 * R * D * I}
    return {"bytes": 2 * (2 * R * D + 3 * busy * D * I), "flops": 6 * R * D * I}


def exact(case, seed):
    if case["op"] in ("route", "slots"):
        return None                                  # whole numbers
    s = prepare(case, seed)
    edges, E, x = s["offsets"].tolist(), case["E"], s["x"].double()
    out = torch.zeros((case["R"], case["N"] if case["op"] == "matvec4" else case["D"]), dtype=torch.float64, device=DEVICE)
    silu = case.get("act", "silu") == "silu"

    def act(a):
        return a / (1 + torch.exp(-a)) if silu else a * torch.special.ndtr(a)

    if case["op"] == "matvec4":
        def weight(part, e):
            q = torch.empty((case["N"], case["K"]), dtype=torch.float64, device=DEVICE)
            q[:, 0::2], q[:, 1::2] = s[part][e] % 16, s[part][e] // 16
            return (q - 8) * s[part + "_scale"][e].double().repeat_interleave(case["group"], 1)

        for e in range(E):
            rows = slice(edges[e], edges[e + 1])
            y = torch.einsum("rk,nk->rn", x[rows], weight("w", e))
            out[rows] = act(y) * torch.einsum("rk,nk->rn", x[rows], weight("up", e)) if case["gated"] else y
        return out
    grads = {k: torch.zeros(s[w].shape, dtype=torch.float64, device=DEVICE) for k, w in
             (("dw_gate", "w_gate"), ("dw_up", "w_up"), ("dw_down", "w_down"))} if case["train"] else {}
    dx = torch.zeros_like(x) if case["train"] else None
    for e in range(E):
        wg, wu, wd = (s[k][e].double() for k in ("w_gate", "w_up", "w_down"))
        for g in range(e, len(edges) - 1, E):
            rows = slice(edges[g], edges[g + 1])
            a, u = x[rows] @ wg.T, x[rows] @ wu.T
            if not case["train"]:
                out[rows] = (act(a) * u) @ wd.T
                continue
            a.requires_grad_()
            f = act(a)
            dy = s["dy"][rows].double()
            dh = dy @ wd
            (slope,) = torch.autograd.grad(f.sum(), a)      # each value depends on its own argument alone
            f = f.detach()
            da, du = dh * u * slope, dh * f
            out[rows], dx[rows] = (f * u) @ wd.T, da @ wg + du @ wu
            grads["dw_gate"][e] += da.T @ x[rows]
            grads["dw_up"][e] += du.T @ x[rows]
            grads["dw_down"][e] += dy.T @ (f * u)
    return {"y": out, "dx": dx, **grads} if case["train"] else out
