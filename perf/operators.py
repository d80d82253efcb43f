"""The operators of a ternary language-model layer as measured cases: the ternary product with its fused epilogue, the
query / key norm with the rotation, and linear attention with a decay per head (whole prompts, and single tokens).

`run` computes a case in plain torch operations in 32 bits, or, where `own` is true, by the calls a user makes of
paper_1912_02057_b200; `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-6


def listed():
    return [
        # one token through a square projection: what each decoding step does several times per layer
        dict(name="linear token", op="linear", M=1, N=4096, K=4096, act="none", bias=False, residual=True, dtype="bf16"),
        # a batch of decoding sequences through an MLP's first product
        dict(name="linear batch", op="linear", M=48, N=16384, K=4096, act="gelu", bias=True, residual=False, dtype="bf16"),
        # a classifier's 512 -> 1000 layer on an odd number of rows
        dict(name="linear ragged", op="linear", M=777, N=1000, K=512, act="silu", bias=True, residual=False, dtype="fp16"),
        # a prompt through an MLP's second product, added to the fp32 residual stream
        dict(name="linear prompt", op="linear", M=8192, N=4096, K=16384, act="none", bias=True, residual=True, dtype="fp32"),
        # a decoding batch: one new token of each of 32 sequences, grouped keys
        dict(name="rotary step", op="rotary", T=32, Hq=32, Hk=8, D=128, R=128, layout="half", norm=True, dtype="bf16"),
        # a middling fp32 prompt, rotation without norms, interleaved pairs
        dict(name="rotary fp32", op="rotary", T=1111, Hq=16, Hk=16, D=64, R=64, layout="interleaved", norm=False, dtype="fp32"),
        # a long prompt whose heads are rotated in part, as projected: q and k are columns of one matrix
        dict(name="rotary prompt", op="rotary", T=16384, Hq=32, Hk=8, D=128, R=64, layout="half", norm=True, dtype="bf16"),
        # a few short requests of different lengths, prefilled together
        dict(name="prompt ragged", op="prompt", B=5, L=300, H=16, Hk=16, D=64, dtype="bf16", fresh=False),
        # a batch of ordinary prompts, grouped keys
        dict(name="prompt batch", op="prompt", B=8, L=2048, H=32, Hk=8, D=128, dtype="bf16", fresh=True),
        # one long document
        dict(name="prompt long", op="prompt", B=1, L=32768, H=16, Hk=16, D=128, dtype="bf16", fresh=True),
        # one sequence decoding alone
        dict(name="token single", op="token", B=1, H=16, Hk=16, D=128, dtype="bf16", slots=False),
        # a serving batch whose states lie in slots of a pool
        dict(name="token batch", op="token", B=96, H=32, Hk=8, D=128, dtype="bf16", slots=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "rotary", "prompt", "token"])
    dtype = rng.choice(["bf16", "bf16", "fp32", "fp16"])
    if op == "linear":
        while True:
            M, N, K = _log_int(rng, 1, 8192), _log_int(rng, 64, 16384), _log_int(rng, 64, 16384)
            if M * N * K <= 8192 * 4096 * 16384:
                break
        return dict(op=op, M=M, N=N, K=K, act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                    bias=rng.random() < 0.5, residual=rng.random() < 0.5, dtype=dtype)
    if op == "rotary":
        D = rng.choice([64, 96, 128, 256])
        Hk = rng.choice([1, 4, 8, 16])
        Hq = Hk * rng.choice([1, 2, 4])
        T = min(_log_int(rng, 1, 16384), 16384 * 40 * 128 // ((Hq + Hk) * D) // (2 if dtype == "fp32" else 1))
        return dict(op=op, T=T, Hq=Hq, Hk=Hk, D=D, R=rng.choice([D, D, D // 2]), layout=rng.choice(["half", "interleaved"]),
                    norm=rng.random() < 0.75, dtype=dtype)
    D = rng.choice([64, 128])
    Hk = rng.choice([4, 8, 16])
    H = Hk * rng.choice([1, 2, 4])
    if op == "prompt":
        B, L = _log_int(rng, 1, 16), _log_int(rng, 1, 32768)
        while B * L * H * D > 32768 * 16 * 128:
            L = max(1, L * 2 // 3)
        return dict(op=op, B=B, L=L, H=H, Hk=Hk, D=D, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), fresh=rng.random() < 0.5)
    return dict(op=op, B=min(_log_int(rng, 1, 256), 96 * 32 * 128 * 128 // (H * D * D)), H=H, Hk=Hk, D=D, dtype=dtype,
                slots=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- inputs

def _planes(codes):
    """Codes int8 [rows, K] as packed rows: per 128 codes 16 bytes of non-zero bits, then 16 bytes of sign bits."""
    rows, K = codes.shape
    nb = (K + 127) // 128
    c = torch.nn.functional.pad(codes, (0, nb * 128 - K)).view(rows, nb, 16, 8)
    bit = 2 ** torch.arange(8, device=codes.device, dtype=torch.int32)
    plane = [((c != 0) * bit).sum(-1).to(torch.uint8), ((c > 0) * bit).sum(-1).to(torch.uint8)]
    return torch.stack(plane, 2).reshape(rows, nb * 32).contiguous()


def _lengths(B, L):
    """Lengths of B prompts, the longest L, spread down to a token; every fifth request has nothing to add."""
    return [0 if b % 5 == 4 else max(1, L - (L * b) // B) if b % 3 else L for b in range(B)]


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=g, device=dev)  # noqa: E731
    s = dict(case)
    dt = DTYPES[case["dtype"]]
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["x"] = ((rand(M, K) < 0.3).to(torch.int8) - (rand(M, K) < 0.3).to(torch.int8))
        s["w"] = ((rand(N, K) < 0.3).to(torch.int8) - (rand(N, K) < 0.3).to(torch.int8))
        s["x_packed"], s["x_sum"] = _planes(s["x"]), s["x"].sum(1, dtype=torch.int32)
        s["w_packed"], s["w_sum"] = _planes(s["w"]), s["w"].sum(1, dtype=torch.int32)
        s["a_scale"], s["a_offset"] = rand(M) + 0.5, rand(M) * 0.2 - 0.1
        s["w_scale"], s["w_offset"] = (rand(N) + 0.5) / math.sqrt(K), (rand(N) * 0.2 - 0.1) / math.sqrt(K)
        s["bias"] = 0.5 * randn(N) if case["bias"] else None
        s["residual"] = randn(M, N).to(dt) if case["residual"] else None
    elif case["op"] == "rotary":
        T, Hq, Hk, D, R = (case[k] for k in ("T", "Hq", "Hk", "D", "R"))
        qkv = (1.5 * randn(T, (Hq + 2 * Hk) * D)).to(dt)
        s["q"], s["k"] = qkv[:, :Hq * D].view(T, Hq, D), qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
        P = 32768
        freq = 10000.0 ** (-torch.arange(0, R, 2, device=dev, dtype=torch.float64) / R)
        angle = torch.arange(P, device=dev, dtype=torch.float64)[:, None] * freq
        s["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        s["positions"] = torch.randint(0, P, (T,), generator=g, device=dev)
        s["q_weight"], s["k_weight"] = (1 + 0.2 * randn(D), 1 + 0.2 * randn(D)) if case["norm"] else (None, None)
    else:
        B, H, Hk, D = (case[k] for k in ("B", "H", "Hk", "D"))
        lens = _lengths(B, case["L"]) if case["op"] == "prompt" else [1] * B
        T = sum(lens)
        qkv = randn(T, (H + 2 * Hk) * D).to(dt)
        s["q"] = qkv[:, :H * D].view(T, H, D)
        s["k"] = qkv[:, H * D:(H + Hk) * D].view(T, Hk, D)
        s["v"] = qkv[:, (H + Hk) * D:].view(T, Hk, D)
        s["log_decay"] = torch.log1p(-torch.exp2(-4.0 - 5.0 * torch.arange(H, device=dev) / H - 0.5 * rand(H)))
        s["scale"] = 1.0 / math.sqrt(D)
        pool = B
        s["slot"] = None
        if case.get("slots"):
            pool = B + B // 4 + 1
            s["slot"] = torch.randperm(pool, generator=g, device=dev)[:B].to(torch.int32)
        s["state"] = None if case.get("fresh") else 2.0 * randn(pool, H, D, D)
        s["state_out"] = torch.zeros(pool, H, D, D, device=dev)
        if case["op"] == "prompt":
            s["max_len"] = max(lens)
            s["start"] = torch.tensor([sum(lens[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)
    return s


# ---------------------------------------------------------------------------------------------- plain forms

def _act(y, act):
    if act == "relu":
        return y.clamp_min(0)
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    return y * torch.sigmoid(y) if act == "silu" else y


def _plain_linear(s):
    codes = s["x"].float() @ s["w"].float().t()                # whole numbers below 2^24: exact
    y = s["a_scale"][:, None] * (s["w_scale"] * codes + s["w_offset"] * s["x_sum"][:, None])
    y = y + s["a_offset"][:, None] * (s["w_scale"] * s["w_sum"] + s["K"] * s["w_offset"])
    if s["bias"] is not None:
        y = y + s["bias"]
    y = _act(y, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(DTYPES[s["dtype"]])


def _plain_rotary_one(x, weight, s):
    y, R = x.float(), s["R"]
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight
    row = s["table"][s["positions"]][:, None, :]
    cos, sin = row[..., :R // 2], row[..., R // 2:]
    rot, rest = y[..., :R], y[..., R:]
    if s["layout"] == "half":
        a, b = rot[..., :R // 2], rot[..., R // 2:]
        rot = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = rot[..., 0::2], rot[..., 1::2]
        rot = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([rot, rest], -1).to(x.dtype)


def _plain_rotary(s):
    return {"q": _plain_rotary_one(s["q"], s["q_weight"], s), "k": _plain_rotary_one(s["k"], s["k_weight"], s)}


def _plain_token(s):
    G = s["H"] // s["Hk"]
    q = s["q"].float()
    k, v = (s[n].float().repeat_interleave(G, 1) for n in ("k", "v"))
    old = s["state"] if s["slot"] is None else s["state"][s["slot"].long()]
    new = old * torch.exp(s["log_decay"])[None, :, None, None] + k[..., None] * v[..., None, :]
    out = s["scale"] * (q[..., None, :] @ new)[..., 0, :]
    if s["slot"] is None:
        s["state_out"].copy_(new)
    else:
        s["state_out"][s["slot"].long()] = new
    return {"out": out.to(s["q"].dtype), "state": s["state_out"]}


def _plain_prompt(s):
    """All prompts padded to the longest, in chunks of C tokens: scores within a chunk, the chunks' states weighed by their
    distance between chunks."""
    B, H, Hk, D, L, C = s["B"], s["H"], s["Hk"], s["D"], s["max_len"], 128
    dev, G, n = s["q"].device, H // Hk, (s["max_len"] + 127) // 128
    g = s["log_decay"]
    first, lens = s["start"][:-1].long(), (s["start"][1:] - s["start"][:-1]).long()
    t = torch.arange(n * C, device=dev)
    inside = t < lens[:, None]                                                     # [B, n C]
    rows = torch.where(inside, first[:, None] + t, torch.zeros_like(t))
    pick = lambda x: torch.where(inside[..., None, None], x[rows].float(), torch.zeros((), device=dev))  # noqa: E731
    q = pick(s["q"]).view(B, n, C, H, D).permute(0, 3, 1, 2, 4)                    # [B, H, n, C, D]
    k, v = (pick(s[x]).view(B, n, C, Hk, D).permute(0, 3, 1, 2, 4).repeat_interleave(G, 1) for x in ("k", "v"))
    i = torch.arange(C, device=dev)
    gap = i[:, None] - i
    near = torch.where(gap >= 0, torch.exp(gap.clamp_min(0) * g[:, None, None]), torch.zeros((), device=dev))     # [H, C, C]
    out = ((q @ k.transpose(-1, -2)) * near[:, None]) @ v
    parts = (k * torch.exp((C - 1 - i) * g[:, None])[:, None, :, None]).transpose(-1, -2) @ v                     # [B, H, n, D, D]
    j = torch.arange(n, device=dev)
    hop = j[:, None] - 1 - j
    far = torch.where(hop >= 0, torch.exp(C * hop.clamp_min(0) * g[:, None, None]), torch.zeros((), device=dev))  # [H, n, n]
    before = (far @ parts.reshape(B, H, n, D * D)).view(B, H, n, D, D)
    if s["state"] is not None:
        before = before + torch.exp(C * j * g[:, None])[..., None, None] * s["state"][:, :, None]
    out = out + (q @ before) * torch.exp((i + 1) * g[:, None])[:, None, :, None]
    out = (s["scale"] * out).permute(0, 2, 3, 1, 4).reshape(B, n * C, H, D)[inside]
    left = torch.where(inside, lens[:, None] - 1 - t, torch.zeros_like(t))
    weight = torch.where(inside[:, None], torch.exp(left[:, None] * g[:, None]), torch.zeros((), device=dev))     # [B, H, n C]
    end = (k.flatten(2, 3) * weight[..., None]).transpose(-1, -2) @ v.flatten(2, 3)
    if s["state"] is not None:
        end = end + torch.exp(lens[:, None] * g)[..., None, None] * s["state"]
    return {"out": out.to(s["q"].dtype), "state": end}


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    if not own:
        return {"linear": _plain_linear, "rotary": _plain_rotary, "prompt": _plain_prompt, "token": _plain_token}[s["op"]](s)
    import paper_1912_02057_b200 as rtn
    if s["op"] == "linear":
        return rtn.rtn_ternary_linear(s["x_packed"], s["x_sum"], s["w_packed"], s["w_sum"], s["M"], s["N"], s["K"],
                                      s["a_scale"], s["a_offset"], s["w_scale"], s["w_offset"], bias=s["bias"],
                                      activation=getattr(rtn, "ACT_" + s["act"].upper()), residual=s["residual"], dtype=DTYPES[s["dtype"]])
    if s["op"] == "rotary":
        q, k = rtn.rtn_qk_norm_rotary(s["q"], s["k"], s["positions"], s["table"], q_weight=s["q_weight"],
                                      k_weight=s["k_weight"], eps=EPS,
                                      layout=getattr(rtn, "ROTARY_" + s["layout"].upper()))
        return {"q": q, "k": k}
    if s["op"] == "prompt":
        out, state = rtn.rtn_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], s["start"], s["max_len"],
                                             state=s["state"], state_out=s["state_out"], scale=s["scale"])
    else:
        out, state = rtn.rtn_decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"],
                                                  state_out=s["state_out"], slots=s["slot"], scale=s["scale"])
    return {"out": out, "state": state}


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        moved = (M + N) * ((K + 127) // 128 * 32 + 12) + M * N * e * (2 if case["residual"] else 1) + (4 * N if case["bias"] else 0)
        return {"bytes": moved, "flops": 2 * M * N * K}
    if case["op"] == "rotary":
        values = case["T"] * (case["Hq"] + case["Hk"]) * case["D"]
        return {"bytes": 2 * e * values + case["T"] * (4 * case["R"] + 8), "flops": values * (4 + (4 if case["norm"] else 0))}
    B, H, Hk, D = (case[k] for k in ("B", "H", "Hk", "D"))
    T = sum(_lengths(B, case["L"])) if case["op"] == "prompt" else B
    states = B * H * D * D * 4 * (1 if case.get("fresh") else 2)
    # the recurrence itself: a state's update and its product with the query, for each token
    return {"bytes": T * D * e * (2 * H + 2 * Hk) + states, "flops": T * H * D * D * 4}


# ---------------------------------------------------------------------------------------------- definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        if case["M"] * case["N"] * case["K"] > 1 << 40:
            return None
        a = s["x"].double() * s["a_scale"].double()[:, None] + s["a_offset"].double()[:, None]
        w = s["w"].double() * s["w_scale"].double()[:, None] + s["w_offset"].double()[:, None]
        y = a @ w.t()
        if s["bias"] is not None:
            y = y + s["bias"].double()
        if case["act"] == "relu":
            y = torch.maximum(y, torch.zeros_like(y))
        elif case["act"] == "silu":
            y = y / (1 + torch.exp(-y))
        elif case["act"] == "gelu":
            y = y * torch.special.ndtr(y)
        elif case["act"] == "gelu_tanh":
            y = y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        return y if s["residual"] is None else y + s["residual"].double()
    if case["op"] == "rotary":
        R, found = case["R"], {}
        turn = torch.complex(s["table"][s["positions"], :R // 2].double(), s["table"][s["positions"], R // 2:].double())[:, None]
        for name in ("q", "k"):
            y = s[name].double()
            if case["norm"]:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / case["D"] + EPS) * s[name + "_weight"].double()
            else:
                y = y.clone()
            at = (torch.arange(0, R // 2, device="cuda"), torch.arange(R // 2, R, device="cuda")) if case["layout"] == "half" else \
                (torch.arange(0, R, 2, device="cuda"), torch.arange(1, R, 2, device="cuda"))
            z = torch.complex(y[..., at[0]], y[..., at[1]]) * turn
            y[..., at[0]], y[..., at[1]] = z.real, z.imag
            found[name] = y
        return found
    # token by token, all sequences at once
    B, H, Hk, D = (case[k] for k in ("B", "H", "Hk", "D"))
    lens = _lengths(B, case["L"]) if case["op"] == "prompt" else [1] * B
    at = [sum(lens[:b]) for b in range(B)]
    group = torch.arange(H, device="cuda") // (H // Hk)
    keep = torch.exp(s["log_decay"].double())[None, :, None, None]
    rows = s["slot"].long() if s["slot"] is not None else torch.arange(B, device="cuda")
    S = torch.zeros(B, H, D, D, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"][rows].double()
    out = torch.empty(sum(lens), H, D, dtype=torch.float64, device="cuda")
    active, last, mine = None, None, None
    for t in range(max(lens)):
        live = [b for b in range(B) if lens[b] > t]
        if live != last:
            last, active = live, torch.tensor(live, device="cuda")
            first = torch.tensor([at[b] for b in live], device="cuda")
            mine = S[active]
        r = first + t
        k, v, q = s["k"][r].double()[:, group], s["v"][r].double()[:, group], s["q"][r].double()
        mine = mine * keep + torch.einsum("bhi,bhj->bhij", k, v)
        out[r] = torch.einsum("bhi,bhij->bhj", q, mine) * case["D"] ** -0.5
        ending = t + 1
        if any(lens[b] == ending for b in live):
            S[active] = mine
    state = s["state_out"].double()
    state[rows] = S
    return {"out": out, "state": state}
