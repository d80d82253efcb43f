"""The operators of a layer of routed ternary experts as measured cases: the choice of experts with the plan of their rows, the
experts' ternary products, and the norms before and after a block with its gate, its residual and the weighted sum of the experts.

`run` computes a case in plain torch operations in 32 bits (codes and choices, which have to be right next to a border, in 64), or,
where `own` is true, by the calls a user makes of paper_1912_02057_b200; `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-6


def listed():
    return [
        # one new token chooses among 64 experts: what each decoding step does once per layer
        dict(name="route token", op="route", T=1, E=64, k=4, score="softmax", bias=False, groups=1, kept=1, top=1, norm=True, dtype="fp32"),
        # a serving batch, sigmoid scores with a balance bias, half of eight groups kept
        dict(name="route batch", op="route", T=96, E=256, k=8, score="sigmoid", bias=True, groups=8, kept=4, top=2, norm=True, dtype="fp32"),
        # long prompts routed together
        dict(name="route prompt", op="route", T=16384, E=128, k=8, score="softmax", bias=False, groups=1, kept=1, top=1, norm=True, dtype="bf16"),
        # the chosen experts' first product for one token, handed on as codes
        dict(name="experts token", op="experts", T=1, E=64, k=4, N=2048, K=2048, gated=True, act="silu", bias=False, gather=True, out="codes", dtype="fp32"),
        # the same for a decoding batch: every expert has a few rows
        dict(name="experts batch", op="experts", T=48, E=64, k=8, N=2048, K=2048, gated=True, act="silu", bias=False, gather=True, out="codes", dtype="fp32"),
        # few large experts of odd sizes, values instead of codes
        dict(name="experts ragged", op="experts", T=777, E=8, k=2, N=1000, K=520, gated=False, act="gelu", bias=True, gather=True, out="values", dtype="fp16"),
        # prompts through the first product
        dict(name="experts prompt up", op="experts", T=8192, E=64, k=8, N=2048, K=2048, gated=True, act="silu", bias=False, gather=True, out="codes", dtype="fp32"),
        # and through the second, whose rows already lie by expert
        dict(name="experts prompt down", op="experts", T=8192, E=64, k=8, N=2048, K=1024, gated=False, act="none", bias=False, gather=False, out="values", dtype="bf16"),
        # one token: four experts' outputs summed into the residual stream, normed, coded for the next block
        dict(name="norm token", op="norm", T=1, W=2048, k=4, branch="bf16", stream="fp32", post=False, gate="none", scale=False, pre=True, out="codes"),
        # a decoding batch through a gated block with norms on both sides
        dict(name="norm batch", op="norm", T=48, W=4096, k=0, branch="fp16", stream="fp16", post=True, gate="silu", scale=True, pre=True, out="normed"),
        # an odd width, no codes, a sigmoid gate
        dict(name="norm odd", op="norm", T=1111, W=5003, k=0, branch="fp32", stream="fp32", post=False, gate="sigmoid", scale=True, pre=True, out="normed"),
        # prompts: eight experts' outputs per token, norms on both sides, codes
        dict(name="norm prompt", op="norm", T=8192, W=2048, k=8, branch="bf16", stream="fp32", post=True, gate="none", scale=True, pre=True, out="codes"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "experts", "experts", "norm"])
    if op == "route":
        E = rng.choice([8, 16, 60, 64, 128, 160, 256])
        groups = rng.choice([1, 1, 2, 4])
        kept = rng.randint(1, groups)
        k = min(rng.choice([1, 2, 4, 6, 8]), E // groups * kept)
        return dict(op=op, T=min(_log_int(rng, 1, 16384), 16384 * 128 // E), E=E, k=k, score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                    groups=groups, kept=kept, top=rng.choice([1, 2]), norm=rng.random() < 0.75, dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]))
    if op == "experts":
        while True:
            T, E = _log_int(rng, 1, 8192), rng.choice([4, 8, 16, 60, 64])
            k = min(rng.choice([1, 2, 4, 6, 8]), E)
            N, K = _log_int(rng, 64, 4096), _log_int(rng, 64, 4096)
            if T * k * N * K <= 65536 * 2048 * 2048 and E * N * K <= 64 * 2048 * 2048 and T * k * N <= 65536 * 2048:
                break
        out = rng.choice(["codes", "values"])
        return dict(op=op, T=T, E=E, k=k, N=N // 2 * 2, K=K, gated=rng.random() < 0.5, act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                    bias=rng.random() < 0.5, gather=rng.random() < 0.6, out=out, dtype="fp32" if out == "codes" else rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    W, k = _log_int(rng, 64, 16384), rng.choice([0, 0, 1, 2, 4, 8])
    T = max(1, min(_log_int(rng, 1, 8192), 8192 * 2048 * 10 // (W * (max(k, 1) + 4))))
    post, pre = rng.random() < 0.5, rng.random() < 0.75
    return dict(op=op, T=T, W=W, k=k, branch=rng.choice(["bf16", "fp16", "fp32"]), stream=rng.choice(["fp32", "fp32", "bf16", "fp16"]), post=post,
                gate=rng.choice(["none", "none", "linear", "sigmoid", "silu"]), scale=rng.random() < 0.5, pre=pre,
                out=rng.choice(["codes", "normed"]) if pre else "stream")


# ---------------------------------------------------------------------------------------------- inputs

def _planes(codes):
    """Codes int8 [rows, K] as packed rows: per 128 codes 16 bytes of non-zero bits, then 16 bytes of sign bits."""
    rows, K = codes.shape
    nb = (K + 127) // 128
    c = torch.nn.functional.pad(codes, (0, nb * 128 - K)).view(rows, nb, 16, 8)
    bit = 2 ** torch.arange(8, device=codes.device, dtype=torch.uint8)
    plane = [((c != 0) * bit).sum(-1, dtype=torch.uint8), ((c > 0) * bit).sum(-1, dtype=torch.uint8)]
    return torch.stack(plane, 2).reshape(rows, nb * 32).contiguous()


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=g, device=dev)  # noqa: E731
    codes = lambda *s: (rand(*s) < 0.3).to(torch.int8) - (rand(*s) < 0.3).to(torch.int8)  # noqa: E731
    s = dict(case)
    T = case["T"]
    if case["op"] == "route":
        E = case["E"]
        # some experts are asked for more often than others; the bias pulls against that
        s["logits"] = (1.5 * randn(T, E) + 0.5 * randn(E)).to(DTYPES[case["dtype"]])
        s["balance"] = 0.05 * randn(E) if case["bias"] else None
    elif case["op"] == "experts":
        E, k, N, K = (case[n] for n in ("E", "k", "N", "K"))
        R, F = T * k, case["N"] // 2 if case["gated"] else case["N"]
        chosen = (randn(T, E) + 0.5 * randn(E)).topk(k, 1).indices
        order = chosen.flatten().argsort(stable=True)
        counts = torch.bincount(chosen.flatten(), minlength=E)
        s["R"], s["F"], s["most"] = R, F, int(counts.max())
        s["start"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s["tokens"] = (order // k).to(torch.int32) if case["gather"] else None
        M = T if case["gather"] else R
        s["x"], s["w"] = codes(M, K), codes(E, N, K)
        s["x_packed"], s["x_sum"] = _planes(s["x"]), s["x"].sum(1, dtype=torch.int32)
        s["w_packed"], s["w_sum"] = _planes(s["w"].view(E * N, K)), s["w"].sum(2, dtype=torch.int32).view(E * N)
        s["a_scale"], s["a_offset"] = rand(M) + 0.5, rand(M) * 0.2 - 0.1
        s["w_scale"], s["w_offset"] = (rand(E * N) + 0.5) / math.sqrt(K), (rand(E * N) * 0.2 - 0.1) / math.sqrt(K)
        s["bias"] = 0.5 * randn(E * N) if case["bias"] else None
        s["t_lo"], s["t_hi"] = torch.tensor([-0.1], device=dev), torch.tensor([0.25], device=dev)
    else:
        W, k = case["W"], case["k"]
        dt, st = DTYPES[case["branch"]], DTYPES[case["stream"]]
        R = T * max(k, 1)
        s["branch"] = (0.7 * randn(R, W)).to(dt)
        s["place"] = torch.randperm(R, generator=g, device=dev).view(T, k).to(torch.int32) if k else None
        s["weights"] = torch.softmax(randn(T, k), 1) if k else None
        s["residual"] = randn(T, W).to(st)
        s["gate_in"] = randn(T, W).to(dt) if case["gate"] != "none" else None
        s["post_weight"] = 1 + 0.2 * randn(W) if case["post"] else None
        s["norm_weight"] = 1 + 0.2 * randn(W) if case["pre"] else None
        s["residual_scale"] = 0.5 + 0.1 * randn(W) if case["scale"] else None
        s["t_lo"], s["t_hi"] = torch.tensor([-0.5], device=dev), torch.tensor([0.5], device=dev)
    return s


# ---------------------------------------------------------------------------------------------- plain forms

def _best_first(x):
    """Values and indices of the last dimension, largest first, ties by index."""
    return torch.sort(x, dim=-1, descending=True, stable=True)


def _plain_route(s):
    T, E, k, G = s["T"], s["E"], s["k"], s["groups"]
    x = s["logits"].double()
    if s["score"] == "softmax":
        e = torch.exp(x - x.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-x))
    choice = score if s["balance"] is None else score + s["balance"].double()
    if G > 1:
        best, _ = _best_first(choice.view(T, G, E // G))
        _, at = _best_first(best[..., :s["top"]].sum(-1))
        keep = torch.zeros(T, G, dtype=torch.bool, device=x.device).scatter_(1, at[:, :s["kept"]], True)
        choice = torch.where(keep.repeat_interleave(E // G, 1), choice, torch.full((), -math.inf, dtype=torch.float64, device=x.device))
    experts = _best_first(choice)[1][:, :k]
    weights = score.gather(1, experts)
    if s["norm"]:
        weights = weights / weights.sum(1, keepdim=True)
    flat = experts.flatten()
    order = torch.sort(flat, stable=True)[1]
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=x.device)
    start = (flat[:, None] < torch.arange(E + 1, device=x.device)).sum(0)
    i32 = torch.int32
    return {"experts": experts.to(i32), "weights": weights.float(), "start": start.to(i32), "tokens": (order // k).to(i32),
            "place": place.view(T, k).to(i32)}


def _act(y, act):
    if act == "relu":
        return y.clamp_min(0)
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    return y * torch.sigmoid(y) if act == "silu" else y


def _coded(v, lo, hi):
    """Packed codes and their sums of values [rows, F]."""
    c = (v > hi.double()).to(torch.int8) - (v < lo.double()).to(torch.int8)
    return _planes(c), c.sum(1, dtype=torch.int32)


def _plain_experts(s):
    """Each expert's rows padded to the most that one has, as one batch of products."""
    E, N, K, R = s["E"], s["N"], s["K"], s["R"]
    r = torch.arange(R, device=s["x"].device)
    of = (r[:, None] >= s["start"][1:]).sum(1)                                    # a row's expert
    at = of * s["most"] + r - s["start"][of]
    m = r if s["tokens"] is None else s["tokens"].long()
    x = torch.zeros(E * s["most"], K, device=s["x"].device)
    x[at] = s["x"][m].float()
    y = (x.view(E, s["most"], K) @ s["w"].float().transpose(1, 2)).view(E * s["most"], N)[at]     # whole numbers below 2^24: exact
    to = (lambda t: t.double()) if s["out"] == "codes" else (lambda t: t)         # codes are those of the value, next to a border too
    row = lambda n: to(s[n])[m][:, None]  # noqa: E731
    col = lambda n: to(s[n]).view(E, N)[of]  # noqa: E731
    w_scale, w_offset = col("w_scale"), col("w_offset")
    y = row("a_scale") * (w_scale * to(y) + w_offset * row("x_sum")) + row("a_offset") * (w_scale * col("w_sum") + K * w_offset)
    if s["bias"] is not None:
        y = y + col("bias")
    y = _act(y[:, :s["F"]], s["act"]) * y[:, s["F"]:] if s["gated"] else _act(y, s["act"])
    if s["out"] == "codes":
        packed, sums = _coded(y, s["t_lo"], s["t_hi"])
        return {"codes": packed, "sums": sums}
    return {"out": y.to(DTYPES[s["dtype"]])}


def _plain_norm(s):
    wide = torch.float64 if s["out"] == "codes" else torch.float32                # codes are those of the value, next to a border too
    y = s["branch"].to(wide)
    if s["place"] is not None:
        y = (s["weights"].to(wide)[..., None] * y[s["place"].long()]).sum(1)
    if s["post_weight"] is not None:
        y = y / torch.sqrt(y.square().mean(1, keepdim=True) + EPS) * s["post_weight"]
    if s["gate_in"] is not None:
        z = s["gate_in"].to(wide)
        y = y * (z if s["gate"] == "linear" else torch.sigmoid(z) if s["gate"] == "sigmoid" else z * torch.sigmoid(z))
    if s["residual_scale"] is not None:
        y = y * s["residual_scale"]
    h = s["residual"].to(wide) + y
    out = {"stream": h.to(s["residual"].dtype)}
    if s["norm_weight"] is not None:
        n = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * s["norm_weight"]
        if s["out"] == "codes":
            out["codes"], out["sums"] = _coded(n, s["t_lo"], s["t_hi"])
        else:
            out["normed"] = n.to(s["branch"].dtype)
    return out


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    if not own:
        return {"route": _plain_route, "experts": _plain_experts, "norm": _plain_norm}[s["op"]](s)
    import paper_1912_02057_b200 as rtn
    if s["op"] == "route":
        r = rtn.rtn_route_experts(s["logits"], s["k"], score=getattr(rtn, "SCORE_" + s["score"].upper()), bias=s["balance"], groups=s["groups"],
                                  kept_groups=s["kept"], group_top=s["top"], renormalise=s["norm"])
        return {"experts": r.experts, "weights": r.weights, "start": r.start, "tokens": r.tokens, "place": r.place}
    if s["op"] == "experts":
        coded = s["out"] == "codes"
        r = rtn.rtn_ternary_experts(s["x_packed"], s["x_sum"], s["tokens"], s["start"], s["w_packed"], s["w_sum"], s["N"], s["K"],
                                    s["a_scale"], s["a_offset"], s["w_scale"], s["w_offset"], bias=s["bias"],
                                    activation=getattr(rtn, "ACT_" + s["act"].upper()), gated=s["gated"], dtype=DTYPES[s["dtype"]],
                                    t_lo=s["t_lo"] if coded else None, t_hi=s["t_hi"] if coded else None)
        return {"codes": r[0], "sums": r[1]} if coded else {"out": r}
    coded = s["out"] == "codes"
    r = rtn.rtn_block_norm(s["branch"], residual=s["residual"], place=s["place"], weights=s["weights"], post_weight=s["post_weight"],
                           gate=s["gate_in"], gate_kind=getattr(rtn, "GATE_" + ("linear" if s["gate"] == "none" else s["gate"]).upper()),
                           scale=s["residual_scale"], norm_weight=s["norm_weight"], eps=EPS, normed=s["out"] == "normed",
                           t_lo=s["t_lo"] if coded else None, t_hi=s["t_hi"] if coded else None)
    return {"stream": r.stream, **({"codes": r.codes, "sums": r.sums} if coded else {"normed": r.normed} if s["out"] == "normed" else {})}


def _row_bytes(K):
    return (K + 127) // 128 * 32


def work(case):
    T = case["T"]
    if case["op"] == "route":
        E, k = case["E"], case["k"]
        return {"bytes": T * E * BYTES[case["dtype"]] + 16 * T * k + 4 * (E + 1) + (4 * E if case["bias"] else 0), "flops": T * E * (4 + k)}
    if case["op"] == "experts":
        E, N, K, R = case["E"], case["N"], case["K"], T * case["k"]
        F = N // 2 if case["gated"] else N
        used = E if R >= E else R                      # experts that have rows, about
        rows = (T if case["gather"] else R) * (_row_bytes(K) + 12) + (4 * R if case["gather"] else 0)
        written = R * (_row_bytes(F) + 4) if case["out"] == "codes" else R * F * BYTES[case["dtype"]]
        return {"bytes": used * N * (_row_bytes(K) + 12 + (4 if case["bias"] else 0)) + rows + written, "flops": 2 * R * N * K}
    W, k, b, st = case["W"], case["k"], BYTES[case["branch"]], BYTES[case["stream"]]
    moved = T * W * (max(k, 1) * b + 2 * st + (b if case["gate"] != "none" else 0)) + 8 * T * k
    moved += {"codes": T * (_row_bytes(W) + 4), "normed": T * W * b, "stream": 0}[case["out"]]
    return {"bytes": moved, "flops": T * W * (2 * max(k, 1) + 4 * case["post"] + 4 * case["pre"] + 4)}


# ---------------------------------------------------------------------------------------------- definitions in 64 bits

def _exact_codes(v, lo, hi):
    """Packed rows and sums, bit by bit of whole words."""
    rows, n = v.shape
    nb = (n + 127) // 128
    up, down = v > hi.double(), v < lo.double()
    words = torch.zeros(rows, nb, 2, 16, dtype=torch.int64, device=v.device)
    pad = lambda b: torch.nn.functional.pad(b.to(torch.int64), (0, nb * 128 - n)).view(rows, nb, 16, 8)  # noqa: E731
    for j in range(8):
        words[:, :, 0] |= pad(up | down)[..., j] << j
        words[:, :, 1] |= pad(up)[..., j] << j
    return words.view(rows, nb * 32).to(torch.uint8), (up.sum(1) - down.sum(1)).to(torch.int32)


def _exact_act(y, act):
    if act == "relu":
        return torch.maximum(y, torch.zeros_like(y))
    if act == "silu":
        return y / (1 + torch.exp(-y))
    if act == "gelu":
        return y * torch.special.ndtr(y)
    if act == "gelu_tanh":
        return y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return y


def exact(case, seed):
    if case["op"] == "experts" and case["T"] * case["k"] * case["N"] * case["K"] >= 1 << 38:
        return None
    s = prepare(case, seed)
    T = case["T"]
    if case["op"] == "route":
        E, k, G = case["E"], case["k"], case["groups"]
        x = s["logits"].double()
        score = torch.softmax(x, 1) if case["score"] == "softmax" else torch.special.expit(x)
        left = score + (0 if s["balance"] is None else s["balance"].double())
        if G > 1:
            per = left.view(T, G, E // G).clone()
            value = torch.zeros(T, G, dtype=torch.float64, device="cuda")
            for _ in range(min(case["top"], E // G)):
                top = per.max(2)
                value += top.values
                per.scatter_(2, top.indices[..., None], -math.inf)
            kept = torch.zeros(T, G, dtype=torch.bool, device="cuda")
            for _ in range(case["kept"]):
                kept.scatter_(1, value.masked_fill(kept, -math.inf).argmax(1, keepdim=True), True)
            left = left.masked_fill(~kept[..., None].expand(T, G, E // G).reshape(T, E), -math.inf)
        found = []
        for _ in range(k):
            i = torch.where(left == left.amax(1, keepdim=True), torch.arange(E, device="cuda"), E).amin(1, keepdim=True)
            found.append(i)
            left = left.scatter(1, i, -math.inf)
        experts = torch.cat(found, 1)
        weights = score.gather(1, experts)
        if case["norm"]:
            weights = weights / weights.sum(1, keepdim=True)
        rows = [torch.nonzero((experts == e).any(1)).flatten() for e in range(E)]
        start = torch.tensor([0] + [len(r) for r in rows], device="cuda").cumsum(0)
        place = torch.empty_like(experts)
        for e in range(E):
            place[experts == e] = torch.arange(len(rows[e]), device="cuda") + start[e]
        i32 = torch.int32
        return {"experts": experts.to(i32), "weights": weights, "start": start.to(i32), "tokens": torch.cat(rows).to(i32), "place": place.to(i32)}
    if case["op"] == "experts":
        E, N, K, F = case["E"], case["N"], case["K"], s["F"]
        y = torch.empty(s["R"], F, dtype=torch.float64, device="cuda")
        start = s["start"].tolist()
        for e in range(E):
            rows = slice(start[e], start[e + 1])
            m = torch.arange(start[e], start[e + 1], device="cuda") if s["tokens"] is None else s["tokens"][rows].long()
            own_cols = slice(e * N, (e + 1) * N)
            a = s["a_scale"].double()[m, None] * s["x"][m] + s["a_offset"].double()[m, None]
            w = s["w_scale"].double()[own_cols, None] * s["w"][e] + s["w_offset"].double()[own_cols, None]
            z = a @ w.t()
            if s["bias"] is not None:
                z = z + s["bias"].double()[own_cols]
            y[rows] = _exact_act(z[:, :F], case["act"]) * z[:, F:] if case["gated"] else _exact_act(z, case["act"])
        if case["out"] == "codes":
            packed, sums = _exact_codes(y, s["t_lo"], s["t_hi"])
            return {"codes": packed, "sums": sums}
        return {"out": y}
    y = s["branch"].double()
    if s["place"] is not None:
        y = sum(s["weights"][:, j, None].double() * s["branch"][s["place"][:, j].long()].double() for j in range(case["k"]))
    if s["post_weight"] is not None:
        y = y * torch.rsqrt((y * y).sum(1, keepdim=True) / case["W"] + EPS) * s["post_weight"].double()
    if s["gate_in"] is not None:
        z = s["gate_in"].double()
        y = y * {"linear": z, "sigmoid": torch.special.expit(z), "silu": z / (1 + torch.exp(-z))}[case["gate"]]
    h = s["residual"].double() + (y if s["residual_scale"] is None else y * s["residual_scale"].double())
    out = {"stream": h}
    if s["norm_weight"] is not None:
        n = h * torch.rsqrt((h * h).sum(1, keepdim=True) / case["W"] + EPS) * s["norm_weight"].double()
        if case["out"] == "codes":
            out["codes"], out["sums"] = _exact_codes(n, s["t_lo"], s["t_hi"])
        else:
            out["normed"] = n
    return out
