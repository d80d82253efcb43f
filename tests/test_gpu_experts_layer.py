"""A layer of routed experts: every stage of its chain against the plain form on the stage's own inputs, for prompts and for single tokens; captured."""
import numpy as np
import pytest
import torch

import paper_1912_02057_b200 as rtn
from paper_1912_02057_b200.decoder import ExpertsLayer, random_experts_layer
import experts_reference as xref
import layer_reference as ref

pytestmark = pytest.mark.gpu


def unpack(packed, n):
    p = packed.cpu().numpy().reshape(packed.shape[0], -1, 2, 16)
    bits = np.unpackbits(p, axis=3, bitorder="little").transpose(2, 0, 1, 3).reshape(2, packed.shape[0], -1)[:, :, :n].astype(np.int8)
    return np.where(bits[0] == 0, 0, 2 * bits[1] - 1).astype(np.int8)


def check(params, trace, x1, k):
    """trace: the layer's intermediate tensors; x1: the stream behind it."""
    x = ref.f64(trace["mlp_in"])
    T, W = x.shape
    f32 = lambda t: tuple(float(np.float32(v)) for v in t)  # noqa: E731
    _, _, n, _ = xref.block_norm(None, x, pre=params["pre_weight"].astype(np.float64))
    codes = xref.codes_of(n, *f32(params["thresholds"]["experts"]))
    assert np.array_equal(trace["mlp_codes"].cpu().numpy(), xref.pack(codes))
    p = params["router"]
    want, mag = ref.linear(codes, p["codes"], [1.0], [0.0], p["scale"], p["offset"], p["bias"])
    ref.assert_close(trace["logits"], want, mag, 24, "logits")
    r = trace["routing"]
    experts, weights, start, tokens, place = xref.route(ref.f64(trace["logits"]), k)
    for got, exact in ((r.experts, experts), (r.start, start), (r.tokens, tokens), (r.place, place)):
        assert np.array_equal(got.cpu().numpy(), exact)
    ref.assert_close(r.weights, weights, weights, 78, "weights")
    one, zero = np.ones(T, np.float32), np.zeros(T, np.float32)
    up = params["expert_up"]
    want, _, live = xref.experts(codes, tokens, start, up["codes"], one, zero, up["scale"], up["offset"], None, rtn.ACT_SILU, True)
    hidden = xref.codes_of(want, *f32(params["thresholds"]["expert_down"]))
    assert live.all() and np.array_equal(trace["hidden"].cpu().numpy(), xref.pack(hidden))
    assert np.array_equal(trace["hidden_sums"].cpu().numpy(), hidden.sum(1, dtype=np.int32))
    down = params["expert_down"]
    one, zero = np.ones(T * k, np.float32), np.zeros(T * k, np.float32)
    want, mag, _ = xref.experts(hidden, np.arange(T * k), start, down["codes"], one, zero, down["scale"], down["offset"])
    ref.assert_close(trace["expert_out"], want, mag, 24, "experts' outputs")
    h, mag, _, _ = xref.block_norm(ref.f64(trace["expert_out"]), x, place, ref.f64(r.weights), params["post_weight"].astype(np.float64),
                                   scale=params["residual_scale"].astype(np.float64))
    ref.assert_close(x1, h, mag, 104, "stream")


@pytest.mark.parametrize("heads,kv_heads,D,width,hidden,experts,k", [(4, 2, 64, 200, 72, 5, 2), (2, 1, 128, 256, 192, 16, 4)])
def test_prompts_then_tokens(heads, kv_heads, D, width, hidden, experts, k):
    params = random_experts_layer(5, width, heads, kv_heads, D, hidden, experts)
    layer = ExpertsLayer(params, rtn.rtn_rotary_table(400, D), top_k=k)
    lens = [150, 1, 37]
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    states = layer.new_states(3)
    x = torch.randn(sum(lens), width, generator=torch.Generator().manual_seed(1)).cuda()
    trace = {}
    y = layer.prompt(x, torch.cat([torch.arange(n) for n in lens]).cuda(), torch.from_numpy(start).cuda(), max(lens), states, trace=trace)
    assert y is x
    check(params, trace, x, k)
    tokens = x[torch.from_numpy(start[1:] - 1).long().cuda()].contiguous()
    for i in range(2):
        trace = {}
        layer.step(tokens, torch.tensor([n + i for n in lens], device="cuda"), states, trace=trace)
        check(params, trace, tokens, k)
    assert rtn.rtn_last_device_status() == 0


def test_a_captured_step_is_the_step():
    params = random_experts_layer(7, 256, 2, 1, 64, 128, 8)
    layer = ExpertsLayer(params, rtn.rtn_rotary_table(64, 64), top_k=2)
    states, at = layer.new_states(40), torch.arange(40, device="cuda") % 64
    given = torch.randn(40, 256, generator=torch.Generator().manual_seed(2)).cuda()
    want, want_states = given.clone(), states.clone()
    layer.step(want, at, want_states)                        # (sets kernel attributes, too)
    x = given.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        layer.step(x, at, states)
    for _ in range(2):
        x.copy_(given)
        states.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want) and torch.equal(states, want_states)
    assert rtn.rtn_last_device_status() == 0


def test_the_example_command_runs_with_experts(capsys, monkeypatch):
    from paper_1912_02057_b200 import decoder
    monkeypatch.setattr("sys.argv", ["decoder", "--layers", "1", "--width", "256", "--hidden", "512", "--heads", "2", "--kv-heads", "1", "--sequences", "3",
                                     "--prompt", "40", "--tokens", "2", "--experts", "8", "--top-k", "2"])
    decoder.main()
    assert "new tokens/s" in capsys.readouterr().out
