"""A decoder layer of a ternary language model as a chain of library calls: every matrix product is ternary x ternary, the sequence is
mixed by linear attention with a decay per head, and the fp32 residual stream is what connects the parts.

    c  = codes of x against the layer's thresholds
    q, k, v = linear(c) (bf16);  q, k <- norm and rotation by position, in place
    x <- x + linear(codes of attention(q, k, v))
    x <- x + linear(codes of act(linear(codes of x)))

or, in a layer of routed experts (`ExpertsLayer`), in place of the last line

    c = codes of norm(x);  experts and weights of each token from linear(c)
    x <- x + scale norm(sum of weight * linear_e(codes of act(gate_e(c)) * up_e(c)))

Prompts go through `prompt` (sequences of different lengths laid end to end), then one token of each sequence at a time through `step`;
the states of all sequences stay in one pool of slots.  Sequencing and argument marshalling only; every operator runs in the
library's kernels.  `python -m paper_1912_02057_b200.decoder` runs a small stack and prints its token rates.
"""
import argparse

import numpy as np
import torch

from . import binding as rtn


def random_layer(seed, width, heads, kv_heads, head_dim, hidden):
    """Seeded random parameters of one layer, as numpy arrays."""
    g = np.random.default_rng(seed)

    def linear(n, k):
        return dict(codes=g.choice(np.array([-1, 0, 1], np.int8), size=(n, k), p=[0.3, 0.4, 0.3]),
                    scale=(g.uniform(0.5, 1.5, n) / np.sqrt(k)).astype(np.float32), offset=np.zeros(n, np.float32),
                    bias=(0.1 * g.normal(size=n)).astype(np.float32))

    return dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                qkv=linear((heads + 2 * kv_heads) * head_dim, width), out=linear(width, heads * head_dim),
                up=linear(hidden, width), down=linear(width, hidden),
                q_weight=g.uniform(0.8, 1.2, head_dim).astype(np.float32), k_weight=g.uniform(0.8, 1.2, head_dim).astype(np.float32),
                log_decay=np.log1p(-np.exp2(-4.0 - 5.0 * np.arange(heads) / heads)).astype(np.float32),
                # thresholds of the ternarizers in front of the four products: (lower, upper)
                thresholds=dict(qkv=(-0.5, 0.5), out=(-0.3, 0.3), up=(-0.5, 0.5), down=(-0.1, 0.4)))


def random_experts_layer(seed, width, heads, kv_heads, head_dim, hidden, experts):
    """The same with `experts` experts of `hidden` values each in place of the dense part."""
    p = random_layer(seed, width, heads, kv_heads, head_dim, width)
    g = np.random.default_rng(seed + 1000)

    def linears(n, k):
        return dict(codes=g.choice(np.array([-1, 0, 1], np.int8), size=(experts, n, k), p=[0.3, 0.4, 0.3]),
                    scale=(g.uniform(0.5, 1.5, (experts, n)) / np.sqrt(k)).astype(np.float32), offset=np.zeros((experts, n), np.float32))

    p["router"] = dict(codes=g.choice(np.array([-1, 0, 1], np.int8), size=(experts, width), p=[0.3, 0.4, 0.3]),
                       scale=(2.0 / np.sqrt(width) * np.ones(experts)).astype(np.float32), offset=np.zeros(experts, np.float32),
                       bias=(0.1 * g.normal(size=experts)).astype(np.float32))
    p["expert_up"], p["expert_down"] = linears(2 * hidden, width), linears(width, hidden)      # (gate rows, then up rows)
    p["pre_weight"], p["post_weight"] = (g.uniform(0.8, 1.2, width).astype(np.float32) for _ in range(2))
    p["residual_scale"] = np.full(width, 0.5, np.float32)
    p["thresholds"].update(experts=(-0.5, 0.5), expert_down=(-0.1, 0.2))
    return p


class DecoderLayer:
    """Device-resident parameters of one layer."""

    products = ("qkv", "out", "up", "down")

    def __init__(self, params, table, activation=rtn.ACT_GELU, eps=1e-6):
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.H, self.Hk, self.D = params["heads"], params["kv_heads"], params["head_dim"]
        self.table, self.activation, self.eps = table, activation, eps
        self.linears = {}
        for name in self.products:
            p = params[name]
            packed, sums = rtn.rtn_pack_weights(dev(p["codes"]))
            lo, hi = params["thresholds"].get(name, (0.0, 0.0))
            self.linears[name] = dict(packed=packed, sums=sums[0], N=p["codes"].shape[0], K=p["codes"].shape[1], scale=dev(p["scale"]),
                                      offset=dev(p["offset"]), bias=dev(p["bias"]), lo=torch.tensor([lo], device="cuda"),
                                      hi=torch.tensor([hi], device="cuda"))
        self.one, self.zero = torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")
        self.q_weight, self.k_weight, self.log_decay = dev(params["q_weight"]), dev(params["k_weight"]), dev(params["log_decay"])

    def _linear(self, name, x, trace, **extra):
        """Codes of x (fp32 [M,K]) through one of the layer's products."""
        p = self.linears[name]
        codes, sums = rtn.rtn_ternarize_pack_act(x, p["lo"], p["hi"])
        if trace is not None:
            trace[name + "_in"] = x.clone()
        y = rtn.rtn_ternary_linear(codes, sums, p["packed"], p["sums"], x.shape[0], p["N"], p["K"], self.one, self.zero, p["scale"],
                                   p["offset"], bias=p["bias"], **extra)
        if trace is not None:
            trace[name + "_out"] = y.clone()
        return y

    def _forward(self, x, positions, attend, trace):
        T, H, Hk, D = x.shape[0], self.H, self.Hk, self.D
        qkv = self._linear("qkv", x, trace, dtype=torch.bfloat16).view(T, H + 2 * Hk, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        rtn.rtn_qk_norm_rotary(q, k, positions, self.table, self.q_weight, self.k_weight, eps=self.eps, out_q=q, out_k=k)
        o = attend(q, k, v)
        if trace is not None:
            trace.update(q=q.clone(), k=k.clone(), v=v.clone(), o=o.clone())
        self._linear("out", o.reshape(T, H * D).float(), trace, residual=x, out=x)
        return self._mlp(x, trace)

    def _mlp(self, x, trace):
        h = self._linear("up", x, trace, activation=self.activation)
        return self._linear("down", h, trace, residual=x, out=x)

    def new_states(self, slots):
        return torch.zeros((slots, self.H, self.D, self.D), dtype=torch.float32, device="cuda")

    def prompt(self, x, positions, start, max_len, states, slots=None, fresh=True, trace=None):
        """x: fp32 [total, width], changed in place; positions int64 [total]; start int32 [B+1]; states of the sequences' slots are
        written (and, unless fresh, read).  trace: optional dict that receives the intermediate tensors."""
        attend = lambda q, k, v: rtn.rtn_decay_attention(q, k, v, self.log_decay, start, max_len, state=None if fresh else states,  # noqa: E731
                                                         state_out=states, slots=slots)[0]
        return self._forward(x, positions, attend, trace)

    def step(self, x, positions, states, slots=None, trace=None):
        """One token of each sequence: x fp32 [B, width], changed in place; states are updated in place."""
        attend = lambda q, k, v: rtn.rtn_decay_attention_step(q, k, v, self.log_decay, states, slots=slots)[0]  # noqa: E731
        return self._forward(x, positions, attend, trace)


class ExpertsLayer(DecoderLayer):
    """A layer whose dense part is `experts` experts, `top_k` of them to a token (parameters: random_experts_layer)."""

    products = ("qkv", "out", "router")

    def __init__(self, params, table, top_k=2, activation=rtn.ACT_SILU, eps=1e-6):
        super().__init__(params, table, activation, eps)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.top_k = top_k
        self.experts = {}
        for name in ("expert_up", "expert_down"):
            p = params[name]
            E, N, K = p["codes"].shape
            packed, sums = rtn.rtn_pack_weights(dev(p["codes"].reshape(E * N, K)))
            self.experts[name] = dict(packed=packed, sums=sums[0], N=N, K=K, scale=dev(p["scale"].reshape(-1)), offset=dev(p["offset"].reshape(-1)))
        self.pre_weight, self.post_weight, self.residual_scale = (dev(params[n]) for n in ("pre_weight", "post_weight", "residual_scale"))
        self.lo, self.hi, self.hidden_lo, self.hidden_hi = (torch.tensor([t], device="cuda") for t in
                                                            (*params["thresholds"]["experts"], *params["thresholds"]["expert_down"]))

    def _experts(self, name, codes, sums, tokens, start, **extra):
        p = self.experts[name]
        return rtn.rtn_ternary_experts(codes, sums, tokens, start, p["packed"], p["sums"], p["N"], p["K"], self.one, self.zero, p["scale"], p["offset"],
                                       **extra)

    def _mlp(self, x, trace):
        before = rtn.rtn_block_norm(None, residual=x, norm_weight=self.pre_weight, eps=self.eps, out=x, t_lo=self.lo, t_hi=self.hi)
        p = self.linears["router"]
        logits = rtn.rtn_ternary_linear(before.codes, before.sums, p["packed"], p["sums"], x.shape[0], p["N"], p["K"], self.one, self.zero,
                                        p["scale"], p["offset"], bias=p["bias"])
        r = rtn.rtn_route_experts(logits, self.top_k)
        hidden, hidden_sums = self._experts("expert_up", before.codes, before.sums, r.tokens, r.start, activation=self.activation, gated=True,
                                            t_lo=self.hidden_lo, t_hi=self.hidden_hi)
        y = self._experts("expert_down", hidden, hidden_sums, None, r.start, dtype=torch.bfloat16)
        if trace is not None:
            trace.update(mlp_in=x.clone(), mlp_codes=before.codes, mlp_sums=before.sums, logits=logits, routing=r, hidden=hidden, hidden_sums=hidden_sums,
                         expert_out=y)
        rtn.rtn_block_norm(y, residual=x, place=r.place, weights=r.weights, post_weight=self.post_weight, scale=self.residual_scale, eps=self.eps, out=x)
        return x


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=8192)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--experts", type=int, default=0, help="routed experts of hidden / 4 values each in place of the dense part")
    ap.add_argument("--top-k", type=int, default=4)
    a = ap.parse_args()
    D = 128
    table = rtn.rtn_rotary_table(a.prompt + a.tokens, D)
    if a.experts:
        layers = [ExpertsLayer(random_experts_layer(i, a.width, a.heads, a.kv_heads, D, a.hidden // 4, a.experts), table, min(a.top_k, a.experts))
                  for i in range(a.layers)]
    else:
        layers = [DecoderLayer(random_layer(i, a.width, a.heads, a.kv_heads, D, a.hidden), table) for i in range(a.layers)]
    states = [l.new_states(a.sequences) for l in layers]
    lens = [max(1, a.prompt * (i + 1) // a.sequences) for i in range(a.sequences)]
    start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    position = torch.cat([torch.arange(n) for n in lens]).cuda()
    x0 = torch.randn(sum(lens), a.width, device="cuda")
    begin, mid, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
    for timed in (False, True):                                  # the first round loads and sets up
        x = x0.clone()
        begin.record()
        for l, s in zip(layers, states):
            l.prompt(x, position, start, max(lens), s)
        mid.record()
        x = x[start[1:].long() - 1].contiguous()
        at = torch.tensor(lens, device="cuda")
        for _ in range(a.tokens):
            for l, s in zip(layers, states):
                l.step(x, at, s)
            at = at + 1
        end.record()
        torch.cuda.synchronize()
    assert rtn.rtn_last_device_status() == 0
    print(f"{a.layers} layers of width {a.width}: {sum(lens) / begin.elapsed_time(mid) * 1e3:.0f} prompt tokens/s "
          f"({a.sequences} prompts, {sum(lens)} tokens), {a.sequences * a.tokens / mid.elapsed_time(end) * 1e3:.0f} new tokens/s")


if __name__ == "__main__":
    main()
