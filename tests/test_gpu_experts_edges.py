"""Operators of a layer of experts where their parts meet: tiles in turn, closed gates, rows of nobody, scores that saturate, squares at the ends of fp32."""
import numpy as np
import pytest
import torch

import paper_1912_02057_b200 as rtn

pytestmark = pytest.mark.gpu

ids = lambda v: str(v).replace("torch.", "").replace(" ", "")  # noqa: E731


def codes(g, *shape):
    return torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8)


# ---------------------------------------------------------------------------------------------- tiles in turn

@pytest.mark.parametrize("E,N,K,gated", [(900, 128, 200, True), (400, 640, 130, False), (300, 256, 1100, True)], ids=ids)
def test_experts_of_few_and_of_many_rows_in_turn(E, N, K, gated):
    """Tiles of 5 rows between tiles of many, some twenty to a CTA: the codes of each come together in its own rows, every time."""
    g = torch.Generator(device="cuda").manual_seed(E)
    counts = torch.tensor([5, 290] * (E // 2), device="cuda")
    start = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    R = int(start[-1])
    x, w = codes(g, R, K), codes(g, E, N, K)
    half, one, zero = (torch.tensor([v], device="cuda") for v in (0.5, 1.0, 0.0))
    xp, xs = rtn.rtn_ternarize_pack_act(x.float(), -half, half)
    wp, ws = rtn.rtn_pack_weights(w.view(E * N, K))
    y = torch.cat([x[a:b].float() @ w[e].float().t() for e, (a, b) in enumerate(zip(start[:-1].tolist(), start[1:].tolist()))])    # (exact: whole numbers)
    t = torch.tensor([4.5], device="cuda")
    want = rtn.rtn_ternarize_pack_act(y[:, :N // 2] * y[:, N // 2:] if gated else y, -t, t)
    places = want[0].clone(), want[1].clone()
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(150):
        places[0].fill_(0xff)
        places[1].fill_(-(1 << 30))
        rtn.rtn_ternary_experts(xp, xs, None, start, wp, ws[0].contiguous(), N, K, one, zero, one, zero, gated=gated, t_lo=-t, t_hi=t, out_packed=places[0],
                                out_sum=places[1])
        wrong += (places[0] != want[0]).sum() + (places[1] != want[1]).sum()
    assert int(wrong) == 0
    assert rtn.rtn_last_device_status() == 0


# ---------------------------------------------------------------------------------------------- closed gates

@pytest.mark.parametrize("kind", [rtn.GATE_SIGMOID, rtn.GATE_SILU])
@pytest.mark.parametrize("low,high,hi", [(-2.0, 2.0, 1.0), (-12.0, -4.0, 0.01), (-40.0, -20.0, 1e-9), (-80.0, -40.0, 1e-20), (-87.2, -80.0, 1e-25), (-100.0, -86.0, 1e-12),
                                         (-110.0, -104.0, 1e-8)], ids=ids)
def test_block_norm_codes_of_closed_gates(low, high, hi, kind):
    """Tokens of one value each (one that is too near for fp32 sends a whole token to the exact form), within a hundred steps of a threshold: the
    code is that of the exact value however far the gate is closed."""
    T = 20000
    r = np.random.default_rng(int(-10 * low) + kind)
    hi = float(np.float32(hi))
    z = r.uniform(low, high, T).astype(np.float32)
    z64 = z.astype(np.float64)
    f = np.exp(z64) / (1.0 + np.exp(z64)) * (z64 if kind == rtn.GATE_SILU else 1.0)
    with np.errstate(over="ignore"):
        y = (hi / f * (1.0 + r.integers(-100, 101, T) * 2.0 ** -24)).astype(np.float32)
    y = np.where(np.isfinite(y), y, np.float32(1.0))                        # (SiLU: about z = 0)
    n = y.astype(np.float64) * f                                           # off by some 2^-51
    sure = np.abs(n / hi - 1.0) > 1e-14
    assert sure.mean() > 0.99 and 0.2 < (n > hi).mean() < 0.8
    dev = lambda a: torch.from_numpy(a).cuda()[:, None]  # noqa: E731
    for sign in (1.0, -1.0):
        t = torch.tensor([hi], device="cuda")
        lo, up = (-torch.full_like(t, np.inf), t) if sign > 0 else (-t, torch.full_like(t, np.inf))
        got = rtn.rtn_block_norm(sign * dev(y), gate=dev(z), gate_kind=kind, t_lo=lo, t_hi=up)
        assert np.array_equal(got.sums.cpu().numpy()[sure], (sign * (n > hi)).astype(np.int32)[sure])
    assert rtn.rtn_last_device_status() == 0


def test_block_norm_gates_that_are_shut():
    """Gates whose logistic function is 0 in double too: what is left is the residual, and no token is NaN."""
    for z in (-746.0, -1e4, -3e38):
        y, r = torch.randn(3, 500, device="cuda"), torch.randn(3, 500, device="cuda")
        t = torch.tensor([0.25], device="cuda")
        for kind in (rtn.GATE_SIGMOID, rtn.GATE_SILU):
            got = rtn.rtn_block_norm(y, r, gate=torch.full_like(y, z), gate_kind=kind, t_lo=-t, t_hi=t)
            want = rtn.rtn_ternarize_pack_act(r, -t, t)
            assert torch.equal(got.stream, r) and torch.equal(got.codes, want[0]) and torch.equal(got.sums, want[1])


# ---------------------------------------------------------------------------------------------- rows of nobody

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
@pytest.mark.parametrize("W", [256, 130, 1003])
def test_block_norm_without_any_rows(W, dtype):
    """No expert has a row: the sum is 0, whatever stands (or does not) where rows would begin; a place that is not negative is out of range."""
    x = torch.randn(5, W, device="cuda")
    weight = 1 + 0.2 * torch.randn(W, device="cuda")
    t = torch.tensor([0.25], device="cuda")
    kw = dict(place=torch.full((5, 3), -1, dtype=torch.int32, device="cuda"), weights=torch.full((5, 3), float("nan"), device="cuda"), post_weight=weight,
              gate=torch.randn(5, W, device="cuda").to(dtype), gate_kind=rtn.GATE_SILU, norm_weight=weight, t_lo=-t, t_hi=t, normed=True)
    want = rtn.rtn_block_norm(None, x, norm_weight=weight, t_lo=-t, t_hi=t, normed=True)
    # an empty tensor of its own, and what is behind the last row of one
    for rows in (torch.empty(0, W, dtype=dtype, device="cuda"), torch.full((1, W), float("nan"), dtype=dtype, device="cuda")[1:]):
        got = rtn.rtn_block_norm(rows, x, **kw)
        assert torch.equal(got.stream, want.stream) and torch.equal(got.normed, want.normed.to(dtype))
        assert torch.equal(got.codes, want.codes) and torch.equal(got.sums, want.sums)
    alone = rtn.rtn_block_norm(torch.empty(0, W, dtype=dtype, device="cuda"), None, place=kw["place"])
    assert alone.stream.dtype == dtype and alone.stream.shape == (5, W) and not bool(alone.stream.any())
    assert rtn.rtn_last_device_status() == 0
    kw["place"][2, 1] = 0
    got = rtn.rtn_block_norm(torch.empty(0, W, dtype=dtype, device="cuda"), x, **kw)
    assert rtn.rtn_last_device_status() == 8 and rtn.rtn_last_device_status() == 0
    keep = [0, 1, 3, 4]
    assert bool(got.stream[2].isnan().all()) and not bool(got.codes[2].any()) and torch.equal(got.stream[keep], want.stream[keep])
    assert torch.equal(got.codes[keep], want.codes[keep])


def test_block_norm_refuses_places_without_choices():
    rows = torch.randn(5, 64, device="cuda")
    for k in (dict(place=torch.empty(5, 0, dtype=torch.int32, device="cuda")), dict(place=torch.empty(5, 0, dtype=torch.int32, device="cuda"),
                                                                                    weights=torch.empty(5, 0, device="cuda"))):
        with pytest.raises(ValueError):
            rtn.rtn_block_norm(rows, rows, **k)


# ---------------------------------------------------------------------------------------------- squares at the ends of fp32

def as_codes(n, lo, hi):
    return np.where(n > hi, 1, np.where(n < lo, -1, 0))


@pytest.mark.parametrize("size", [1e-22, 1e-20, 1e-18, 1e-15, 1e17, 3e17, 1e19])
@pytest.mark.parametrize("W", [256, 131])
def test_block_norm_codes_where_squares_leave_fp32(W, size):
    """Without an epsilon a row's size does not count: the codes are those of the same row at any size, for both norms."""
    T = 3000
    r = np.random.default_rng(W)
    x = (r.standard_normal((T, W)) * size).astype(np.float32)
    x64, weight = x.astype(np.float64), r.uniform(0.8, 1.2, W).astype(np.float32)
    n = x64 / np.sqrt((x64 * x64).mean(1, keepdims=True)) * weight
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    for hi in (0.5, 1.0):
        t = torch.tensor([hi], device="cuda")
        want = as_codes(n, -hi, hi)
        assert np.abs(np.abs(n) - hi).min() > 1e-10              # (no value is nearer than double tells)
        for kw in (dict(branch=None, residual=dev(x), norm_weight=dev(weight)), dict(branch=dev(x), post_weight=dev(weight))):
            got = rtn.rtn_block_norm(**kw, eps=0.0, t_lo=-t, t_hi=t)
            assert np.array_equal(got.sums.cpu().numpy(), want.sum(1))
            p = got.codes.cpu().numpy().reshape(T, -1, 2, 16)
            bits = np.unpackbits(p, axis=3, bitorder="little").transpose(2, 0, 1, 3).reshape(2, T, -1)[:, :, :W]
            assert np.array_equal(bits[0], want != 0) and np.array_equal(bits[1], want > 0)
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("apart", [2.0 ** -23, 2.0 ** -21, 2.0 ** -18, 2.0 ** -12])
@pytest.mark.parametrize("eps", [0.0, 1e-16])
def test_block_norm_codes_of_sums_that_cancel(apart, eps):
    """Two experts' rows that all but cancel: what fp32 leaves of their sum is mostly rounding, and the codes are those of the exact sum all the same."""
    T, W = 2000, 256
    r = np.random.default_rng(5)
    a = r.standard_normal((T, W)).astype(np.float32)
    rows = np.concatenate([a, a * (1.0 + apart * r.integers(-3, 4, (T, W)))]).astype(np.float32)
    w = np.tile(np.float32([0.3, -0.3]), (T, 1)) * r.uniform(1.0, 2.0, (T, 1)).astype(np.float32)
    y = w[:, :1].astype(np.float64) * rows[:T] + w[:, 1:].astype(np.float64) * rows[T:]
    n = y / np.sqrt((y * y).mean(1, keepdims=True) + eps)
    dev = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    place, ones = dev(np.stack([np.arange(T), np.arange(T, 2 * T)], 1).astype(np.int32)), torch.ones(W, device="cuda")
    for hi in (0.05, 0.7, 3.0):
        want = as_codes(n, -float(np.float32(hi)), float(np.float32(hi)))
        t = torch.tensor([hi], device="cuda")
        for norm in ("post_weight", "norm_weight"):
            got = rtn.rtn_block_norm(dev(rows), place=place, weights=dev(w), eps=eps, t_lo=-t, t_hi=t, **{norm: ones})
            assert np.array_equal(got.sums.cpu().numpy(), want.sum(1))
            p = got.codes.cpu().numpy().reshape(T, -1, 2, 16)
            bits = np.unpackbits(p, axis=3, bitorder="little").transpose(2, 0, 1, 3).reshape(2, T, -1)[:, :, :W]
            assert np.array_equal(bits[0], want != 0) and np.array_equal(bits[1], want > 0)


# ---------------------------------------------------------------------------------------------- thresholds the other way round

def plus_first(v, lo, hi):
    """1 above hi, else -1 below lo, else 0, for any lo and hi."""
    return as_codes(v, lo, hi).astype(np.int8)


def packed_of(c):
    rows, n = c.shape
    p = np.zeros((rows, -(-n // 128) * 128), np.int8)
    p[:, :n] = c
    p = p.reshape(rows, -1, 128)
    return np.concatenate([np.packbits(p != 0, axis=2, bitorder="little"), np.packbits(p > 0, axis=2, bitorder="little")], 2).reshape(rows, -1)


@pytest.mark.parametrize("lo,hi", [(0.5, -0.5), (-0.25, -0.75), (0.75, 0.25), (0.5, 0.5), (float("inf"), float("-inf")), (0.0, 0.0)], ids=ids)
@pytest.mark.parametrize("R", [5, 600])
def test_codes_of_thresholds_that_overlap(R, lo, hi):
    """Few rows and many through the experts, every activation that leaves whole sums exact; and the norms."""
    g = torch.Generator(device="cuda").manual_seed(R)
    E, N, K = 3, 200, 90
    x, w = codes(g, R, K), codes(g, E, N, K)
    start = torch.tensor([0, R // 3, R // 3, R], dtype=torch.int32, device="cuda")
    half, one, zero, step = (torch.tensor([v], device="cuda") for v in (0.5, 1.0, 0.0, 0.25))
    xp, xs = rtn.rtn_ternarize_pack_act(x.float(), -half, half)
    wp, ws = rtn.rtn_pack_weights(w.view(E * N, K))
    of = np.repeat([0, 2], [R // 3, R - R // 3])
    y = 0.25 * np.stack([w[e].cpu().numpy().astype(np.float64) @ v for e, v in zip(of, x.cpu().numpy().astype(np.float64))])    # (multiples of 1/4: exact)
    t = dict(t_lo=torch.tensor([lo], device="cuda"), t_hi=torch.tensor([hi], device="cuda"))
    for act in (rtn.ACT_NONE, rtn.ACT_RELU):
        z = y if act == rtn.ACT_NONE else np.maximum(y, 0.0)
        first = np.maximum(y[:, :N // 2], 0.0) if act == rtn.ACT_RELU else y[:, :N // 2]
        for gated in (False, True):
            want = plus_first(first * y[:, N // 2:] if gated else z, lo, hi)
            got = rtn.rtn_ternary_experts(xp, xs, None, start, wp, ws[0].contiguous(), N, K, one, zero, step, zero, activation=act, gated=gated, **t)
            assert np.array_equal(got[0].cpu().numpy(), packed_of(want)) and np.array_equal(got[1].cpu().numpy(), want.sum(1))
    for W in (256, 130, 131):
        v = 0.25 * torch.randint(-6, 7, (R, W), generator=g, device="cuda").float()
        want = plus_first(v.cpu().numpy(), lo, hi)
        got = rtn.rtn_block_norm(None, v, **t)
        assert np.array_equal(got.codes.cpu().numpy(), packed_of(want)) and np.array_equal(got.sums.cpu().numpy(), want.sum(1))
        per = rtn.rtn_block_norm(None, v, t_lo=t["t_lo"].expand(W).contiguous(), t_hi=t["t_hi"].expand(W).contiguous())
        assert torch.equal(got.codes, per.codes) and torch.equal(got.sums, per.sums)
    assert rtn.rtn_last_device_status() == 0


# ---------------------------------------------------------------------------------------------- other streams

def layer(seed, T, E=12, W=256, H=128, k=3):
    """A chain of the operators, whose inputs are all there before its first call."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, logits = randn(T, W), randn(T, E)
    up, us = rtn.rtn_pack_weights(codes(g, E * 2 * H, W))
    down, ds = rtn.rtn_pack_weights(codes(g, E * W, H))
    us, ds = us[0].contiguous(), ds[0].contiguous()
    one, zero, small, lo, hi, low, high = (torch.tensor([v], device="cuda") for v in (1.0, 0.0, 0.05, -0.4, 0.4, -0.1, 0.1))
    weight = 1 + 0.1 * randn(W)

    def run(stream=None):
        n = rtn.rtn_block_norm(None, x, norm_weight=weight, t_lo=lo, t_hi=hi, stream=stream)
        r = rtn.rtn_route_experts(logits, k, stream=stream)
        h = rtn.rtn_ternary_experts(n.codes, n.sums, r.tokens, r.start, up, us, 2 * H, W, one, zero, small, zero, activation=rtn.ACT_SILU, gated=True,
                                    t_lo=low, t_hi=high, stream=stream)
        y = rtn.rtn_ternary_experts(h[0], h[1], None, r.start, down, ds, W, H, one, zero, small, zero, dtype=torch.bfloat16, stream=stream)
        z = rtn.rtn_block_norm(y, x, place=r.place, weights=r.weights, post_weight=weight, norm_weight=weight, normed=True, t_lo=lo, t_hi=hi, stream=stream)
        return [n.codes, n.sums, *r, *h, y, *z]
    return run


@pytest.mark.parametrize("sizes", [(1, 5), (700, 900), (2, 5000), (100, 16000)], ids=str)
def test_two_streams_at_a_time_in_memory_of_earlier_results(sizes):
    """Twenty layers on each of two streams, four times; in between the results' memory is filled with something else."""
    chains = [layer(i, T) for i, T in enumerate(sizes)]
    want = [[t.clone() for t in run()] for run in chains]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in chains]
    for fill in (0x11, 0xa5, 0x11, 0xff):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        got = [[run(stream=s) for run, s in zip(chains, streams)] for _ in range(20)]
        torch.cuda.synchronize()
        for both in got:
            for a, b in zip(both, want):
                assert all(torch.equal(p, q) for p, q in zip(a, b))
        for t in (t for both in got for a in both for t in a):
            t.view(torch.uint8).fill_(fill)
        torch.cuda.synchronize()
        del got, both, a
    assert rtn.rtn_last_device_status() == 0


def calls_with_temporaries():
    """Name and call of each layer operator, on tensors that are made for the call and let go of behind it."""
    g = torch.Generator(device="cuda").manual_seed(3)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    T, W, E, D = 70, 256, 8, 64
    x, logits, half, zero = randn(T, W), randn(T, E), torch.tensor([0.5], device="cuda"), torch.zeros(1, device="cuda")
    xp, xs = rtn.rtn_ternarize_pack_act(x, -half, half)
    wp, ws = rtn.rtn_pack_weights(codes(g, E * W, W))
    ws = ws[0].contiguous()
    table, q, kv, decay, weight = rtn.rtn_rotary_table(300, D), randn(T, 4, D), randn(T, 2, D), -0.1 * torch.ones(4, device="cuda"), randn(W)
    route = rtn.rtn_route_experts(logits, 2)
    rows = randn(2 * T, W)
    states = randn(T, 4, D, D)
    one = half + half
    return [("linear", lambda on: [rtn.rtn_ternary_linear(xp + 0, xs + 0, wp[:W] + 0, ws[:W] + 0, T, W, W, one + 0, zero + 0, one + 0, zero + 0, bias=weight + 0, residual=x + 0,
                                                          stream=on)]),
            ("rotary", lambda on: [t for t in rtn.rtn_qk_norm_rotary(q + 0, kv + 0, torch.arange(T, device="cuda"), table + 0, weight[:D] + 0, weight[:D] + 0, stream=on)]),
            ("prompt", lambda on: rtn.rtn_decay_attention(q + 0, kv + 0, kv + 0, decay + 0, torch.tensor([0, 30, T], dtype=torch.int32).cuda(), 40, stream=on)),
            ("step", lambda on: rtn.rtn_decay_attention_step(q + 0, kv + 0, kv + 0, decay + 0, states + 0, stream=on)),
            ("route", lambda on: rtn.rtn_route_experts(logits + 0, 3, score=rtn.SCORE_SIGMOID, bias=logits[0] + 0, stream=on)),
            ("experts", lambda on: rtn.rtn_ternary_experts(xp + 0, xs + 0, route.tokens + 0, route.start + 0, wp + 0, ws + 0, W, W, one + 0, zero + 0, one + 0, zero + 0,
                                                           t_lo=-half, t_hi=half + 0, stream=on)),
            ("norm", lambda on: rtn.rtn_block_norm(rows + 0, x + 0, place=route.place + 0, weights=route.weights + 0, post_weight=weight + 0, gate=x + 0, scale=weight + 0,
                                                   norm_weight=weight + 0, t_lo=-half, t_hi=half + 0, stream=on))]


def test_temporaries_stay_until_the_given_stream_has_used_them():
    side = torch.cuda.Stream()
    for name, call in calls_with_temporaries():
        want = [t.clone() for t in call(None) if t is not None]
        torch.cuda.synchronize()
        for _ in range(2):
            with torch.cuda.stream(side):
                torch.cuda._sleep(20_000_000)
            got = [t for t in call(side) if t is not None]
            # what the temporaries left behind, if anything, goes to these
            junk = [torch.full((n,), 0x7f, dtype=torch.uint8, device="cuda") for n in [1 << b for b in range(2, 23)] + [280, 560, 32, 36, 64, 1024] + [8] * 20]
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got)), name
            del junk
    # with a stream of the caller's that torch does not own, and with the current one
    held = torch.cuda.ExternalStream(side.cuda_stream)
    for name, call in calls_with_temporaries():
        want = [t.clone() for t in call(None) if t is not None]
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            for on in (side, held, None):
                got = [t for t in call(on) if t is not None]
                side.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(want, got)), name
    with pytest.raises(AttributeError):
        rtn.rtn_route_experts(torch.zeros(2, 4, device="cuda"), 1, stream=7)
    assert rtn.rtn_last_device_status() == 0
