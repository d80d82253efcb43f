"""The decoder layer: every stage of its chain against the plain form on the stage's own inputs, for prompts and for single tokens."""
import numpy as np
import pytest
import torch

import paper_1912_02057_b200 as rtn
from paper_1912_02057_b200.decoder import DecoderLayer, random_layer
import layer_reference as ref

pytestmark = pytest.mark.gpu


def codes_of(x, lo, hi):
    return np.where(x > hi, 1, np.where(x < lo, -1, 0)).astype(np.int8)


def check(params, trace, x0, x1, positions, table, start, state, end, act, longest):
    """trace: the layer's intermediate tensors; state, end: the sequences' states before and after (numpy)."""
    H, Hk, D = params["heads"], params["kv_heads"], params["head_dim"]
    T = x0.shape[0]
    n = {k: ref.f64(v) for k, v in trace.items()}
    assert np.array_equal(n["qkv_in"], x0)

    def linear(name, kind=0, residual=None):
        p = params[name]
        lo, hi = (np.float32(t) for t in params["thresholds"][name])
        want, mag = ref.linear(codes_of(n[name + "_in"], lo, hi), p["codes"], [1.0], [0.0], p["scale"], p["offset"], p["bias"], kind, residual)
        ref.assert_close(trace[name + "_out"], want, mag, 24, name)

    linear("qkv")
    qkv = n["qkv_out"].reshape(T, H + 2 * Hk, D)
    for name, part, w in (("q", qkv[:, :H], params["q_weight"]), ("k", qkv[:, H:H + Hk], params["k_weight"])):
        ref.assert_close(trace[name], *ref.rotary(part, positions, table, w, 1e-6, 0), 40, name)
    assert np.array_equal(n["v"], qkv[:, H + Hk:])
    want, mag, want_end, mag_end = ref.decay(n["q"], n["k"], n["v"], params["log_decay"], start, state, D ** -0.5)
    c = ref.decay_roundings(params["log_decay"], longest, D)
    ref.assert_close(trace["o"], want, mag, c, "o", extra=2.0 ** -15)
    ref.assert_close(end, want_end, mag_end, c, "state")
    assert np.array_equal(n["out_in"], n["o"].reshape(T, H * D))
    linear("out", residual=x0)
    assert np.array_equal(n["up_in"], n["out_out"])
    linear("up", kind=act)
    assert np.array_equal(n["down_in"], n["up_out"])
    linear("down", residual=n["out_out"])
    assert np.array_equal(n["down_out"], ref.f64(x1))


@pytest.mark.parametrize("heads,kv_heads,D,width,hidden,act", [(4, 2, 64, 200, 520, rtn.ACT_GELU), (2, 1, 128, 256, 384, rtn.ACT_SILU)])
def test_prompts_then_tokens(heads, kv_heads, D, width, hidden, act):
    params = random_layer(5, width, heads, kv_heads, D, hidden)
    table = rtn.rtn_rotary_table(400, D)
    layer = DecoderLayer(params, table, activation=act)
    lens = [150, 1, 37]
    B = len(lens)
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    positions = np.concatenate([np.arange(n) for n in lens])
    slots = torch.tensor([3, 0, 2], dtype=torch.int32, device="cuda")
    states = layer.new_states(5)
    states[1], states[4] = 7.0, 7.0
    x = torch.randn(sum(lens), width, generator=torch.Generator().manual_seed(1)).cuda()
    x0, trace = ref.f64(x), {}
    y = layer.prompt(x, torch.from_numpy(positions).cuda(), torch.from_numpy(start).cuda(), max(lens), states, slots=slots, trace=trace)
    assert y is x
    check(params, trace, x0, x, positions, ref.f64(table), start, None, states[slots.long()], act, max(lens))
    tokens = x[torch.from_numpy(start[1:] - 1).long().cuda()].contiguous()
    for i in range(3):
        at = np.array(lens) + i
        x0, trace, before = ref.f64(tokens), {}, states[slots.long()].cpu().numpy()
        layer.step(tokens, torch.from_numpy(at).cuda(), states, slots=slots, trace=trace)
        check(params, trace, x0, tokens, at, ref.f64(table), np.arange(B + 1), before, states[slots.long()], act, 1)
    assert bool((states[[1, 4]] == 7.0).all())
    assert rtn.rtn_last_device_status() == 0


def test_the_example_command_runs(capsys, monkeypatch):
    from paper_1912_02057_b200 import decoder
    monkeypatch.setattr("sys.argv", ["decoder", "--layers", "1", "--width", "256", "--hidden", "512", "--heads", "2", "--kv-heads", "1",
                                     "--sequences", "3", "--prompt", "40", "--tokens", "2"])
    decoder.main()
    assert "new tokens/s" in capsys.readouterr().out
