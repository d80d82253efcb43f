"""Operators of a layer of experts where offsets pass 32 bits, and several calls and captured graphs at work at a time."""
import pytest
import torch

import paper_1912_02057_b200 as rtn

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def codes(g, *shape):
    return torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8)


@pytest.mark.parametrize("rows", [6, 3000], ids=["few", "many"])
def test_planes_behind_four_gigabytes(rows):
    """The last of the experts: its planes begin more than 2^32 bytes behind the first's.  The same rows with that expert alone."""
    g = gen(rows)
    E, N, K = 70, 16384, 16384
    nbytes = rtn.rtn_packed_row_bytes(K)
    wp = torch.zeros(E * N, nbytes, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(E * N, dtype=torch.int32, device="cuda")
    assert wp.numel() > 2 ** 32 + N * nbytes
    one_p, one_s = rtn.rtn_pack_weights(codes(g, N, K))
    wp[-N:], ws[-N:] = one_p.view(N, -1), one_s[0]
    half, one, zero = (torch.tensor([v], device="cuda") for v in (0.5, 1.0, 0.0))
    xp, xs = rtn.rtn_ternarize_pack_act(codes(g, rows, K).float(), -half, half)
    start = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    start[-1] = rows
    t = torch.tensor([30.5], device="cuda")
    kw = dict(gated=True, t_lo=-t, t_hi=t)
    alone = (xp, xs, None, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), wp[-N:], ws[-N:].contiguous(), N, K, one, zero, one, zero)
    among = (xp, xs, None, start, wp, ws, N, K, one, zero, one, zero)
    want, got = rtn.rtn_ternary_experts(*alone, **kw), rtn.rtn_ternary_experts(*among, **kw)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and bool(want[0].any())
    assert rtn.rtn_last_device_status() == 0


def test_outputs_and_streams_behind_two_billion_elements():
    g = gen(1)
    E, N, K, T = 2, 16384, 256, 140000
    x, w = codes(g, T, K), codes(g, E * N, K)
    half, one, zero = (torch.tensor([v], device="cuda") for v in (0.5, 1.0, 0.0))
    xp, xs = rtn.rtn_ternarize_pack_act(x.float(), -half, half)
    wp, ws = rtn.rtn_pack_weights(w)
    start = torch.tensor([0, 1000, T], dtype=torch.int32, device="cuda")
    out = rtn.rtn_ternary_experts(xp, xs, None, start, wp, ws[0].contiguous(), N, K, one, zero, one, zero, dtype=torch.bfloat16)
    assert out.numel() > 2 ** 31
    for rows, e in ((slice(0, 100), 0), (slice(T - 300, T), 1)):           # (whole sums up to 256 are exact in bf16)
        assert torch.equal(out[rows].float(), x[rows].float() @ w[e * N:(e + 1) * N].float().t())
    # the same tensor as the rows that a norm adds up and the stream that it goes on with
    place = torch.arange(T, device="cuda", dtype=torch.int32).flip(0).view(T, 1).contiguous()
    weight = 1 + 0.1 * torch.randn(N, generator=g, device="cuda")
    n = rtn.rtn_block_norm(out, out, place=place, post_weight=weight, norm_weight=weight, t_lo=-half, t_hi=half)
    tail = slice(T - 64, T)
    want = rtn.rtn_block_norm(out[place[tail, 0].long()], out[tail], post_weight=weight, norm_weight=weight, t_lo=-half, t_hi=half)
    assert torch.equal(n.codes[tail], want.codes) and torch.equal(n.sums[tail], want.sums) and torch.equal(n.stream[tail], want.stream)
    assert rtn.rtn_last_device_status() == 0


def layer(seed, T, E=12, W=256, H=128, k=3):
    """A chain of the operators with buffers of its own: run() gives its outputs."""
    g = gen(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, logits = randn(T, W), randn(T, E)
    up, us = rtn.rtn_pack_weights(codes(g, E * 2 * H, W))
    down, ds = rtn.rtn_pack_weights(codes(g, E * W, H))
    us, ds = us[0].contiguous(), ds[0].contiguous()
    one, zero, small, t, th = (torch.tensor([v], device="cuda") for v in (1.0, 0.0, 0.05, 0.4, 0.1))
    weight = 1 + 0.1 * randn(W)

    def run(stream=None):
        n = rtn.rtn_block_norm(None, x, norm_weight=weight, t_lo=-t, t_hi=t, stream=stream)
        r = rtn.rtn_route_experts(logits, k, stream=stream)
        hidden = rtn.rtn_ternary_experts(n.codes, n.sums, r.tokens, r.start, up, us, 2 * H, W, one, zero, small, zero, activation=rtn.ACT_SILU, gated=True,
                                         t_lo=-th, t_hi=th, stream=stream)
        y = rtn.rtn_ternary_experts(hidden[0], hidden[1], None, r.start, down, ds, W, H, one, zero, small, zero, dtype=torch.bfloat16, stream=stream)
        z = rtn.rtn_block_norm(y, x, place=r.place, weights=r.weights, post_weight=weight, norm_weight=weight, normed=True, t_lo=-t, t_hi=t, stream=stream)
        return [n.codes, r.experts, r.weights, r.tokens, hidden[0], hidden[1], y, z.stream, z.normed, z.codes, z.sums]
    return x, logits, run


@pytest.mark.parametrize("sizes", [(1, 5), (700, 900), (2, 5000)], ids=str)
def test_two_streams_at_a_time(sizes):
    chains = [layer(i, T) for i, T in enumerate(sizes)]
    want = [[t.clone() for t in run()] for _, _, run in chains]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in chains]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(20):
        got.append([run(stream=s) for (_, _, run), s in zip(chains, streams)])
    torch.cuda.synchronize()
    for both in got:
        for a, b in zip(both, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("sizes", [(1, 5), (700, 900)], ids=str)
def test_two_captured_chains_replayed_at_a_time(sizes):
    chains, graphs, outs = [layer(10 + i, T) for i, T in enumerate(sizes)], [], []
    for _, _, run in chains:
        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in chains]
    g = gen(3)
    for _ in range(5):
        for x, logits, _ in chains:                                       # new inputs at the captured addresses
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            logits.copy_(torch.randn(logits.shape, generator=g, device="cuda"))
        want = [[t.clone() for t in run()] for _, _, run in chains]
        torch.cuda.synchronize()
        for _ in range(3):
            for graph, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("E,R", [(1024, 20000), (1023, 900), (1, 5000), (1, 161)], ids=str)
def test_from_one_to_the_most_experts(E, R):
    """Whole sums against a product in fp32, which is exact; some experts without rows."""
    g = gen(E + R)
    N, K = 200, 300
    x, w = codes(g, R, K), codes(g, E, N, K)
    counts = torch.multinomial(torch.rand(E, generator=g, device="cuda") ** 4 + 1e-6, R, replacement=True, generator=g).bincount(minlength=E)
    start = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    half, one, zero = (torch.tensor([v], device="cuda") for v in (0.5, 1.0, 0.0))
    xp, xs = rtn.rtn_ternarize_pack_act(x.float(), -half, half)
    wp, ws = rtn.rtn_pack_weights(w.view(E * N, K))
    got = rtn.rtn_ternary_experts(xp, xs, None, start, wp, ws[0].contiguous(), N, K, one, zero, one, zero)
    of = torch.repeat_interleave(torch.arange(E, device="cuda"), counts)
    want = torch.cat([torch.bmm(w[of[i:i + 500]].float(), x[i:i + 500].float().unsqueeze(2)).squeeze(2) for i in range(0, R, 500)])
    assert torch.equal(got, want)
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("R", [1, 40])
def test_the_longest_rows(R):
    """K = 2^24: the largest sum that fp32 holds exactly."""
    N, K = 8, 1 << 24
    half, one, zero = (torch.tensor([v], device="cuda") for v in (0.5, 1.0, 0.0))
    x = torch.ones(1, K, device="cuda")
    x[0, 5::7] = -1
    row = [rtn.rtn_ternarize_pack_act(v, -half, half) for v in (torch.ones(1, K, device="cuda"), x)]
    xp = torch.cat([row[i % 2][0].view(1, -1) for i in range(R)])
    xs = torch.cat([row[i % 2][1] for i in range(R)])
    w = torch.ones(N, K, dtype=torch.int8, device="cuda")
    w[1] = -1
    w[2, ::2] = 0
    w[3] = x[0].to(torch.int8)
    wp, ws = rtn.rtn_pack_weights(w)
    got = rtn.rtn_ternary_experts(xp, xs, None, torch.tensor([0, R], dtype=torch.int32, device="cuda"), wp, ws[0].contiguous(), N, K, one, zero, one, zero)
    minus = len(range(5, K, 7))
    first = torch.tensor([K, -K, K // 2, K - 2 * minus] + [K] * 4, dtype=torch.float64)
    odd = sum(1 for _ in range(5, K, 14))                                   # the minus ones at odd places: 5, 19, 33, ...
    second = torch.tensor([K - 2 * minus, 2 * minus - K, K // 2 - 2 * odd, K] + [K - 2 * minus] * 4, dtype=torch.float64)
    want = torch.stack([(first, second)[i % 2] for i in range(R)])
    assert torch.equal(got.double().cpu(), want)
    assert rtn.rtn_last_device_status() == 0


def joined(T, W, E):
    """Inputs that two streams make, each at the end of long work of its own, then the operators at once."""
    g = gen(T)
    base = torch.randn(T, W, generator=g, device="cuda")
    big = torch.randn(2048, 2048, generator=g, device="cuda")
    up, us = rtn.rtn_pack_weights(codes(g, E * W, W))
    us = us[0].contiguous()
    one, zero, t = (torch.tensor([v], device="cuda") for v in (1.0, 0.0, 0.4))
    side = torch.cuda.Stream()
    x, r, logits = torch.empty_like(base), torch.empty_like(base), torch.empty(T, E, device="cuda")
    scale = torch.ones((), device="cuda")

    def slow(v, out):
        y = big
        for _ in range(6):
            y = (y @ big) * 1e-2
        torch.mul(v, scale + 0 * y[0, 0], out=out)

    def run():
        main = torch.cuda.current_stream()
        for t_ in (x, r, logits):
            t_.fill_(float("nan"))
        side.wait_stream(main)
        with torch.cuda.stream(side):
            slow(base.flip(0), r)
        slow(base, x)
        torch.mul(x[:, :E], 2.0, out=logits)
        main.wait_stream(side)
        n = rtn.rtn_block_norm(x, r, norm_weight=torch.ones(W, device="cuda"), t_lo=-t, t_hi=t)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            slow(base[:, :E], logits)
        main.wait_stream(side)
        route = rtn.rtn_route_experts(logits, 2)
        main.wait_stream(side)
        y = rtn.rtn_ternary_experts(n.codes, n.sums, route.tokens, route.start, up, us, W, W, one, zero, one, zero, t_lo=-t, t_hi=t)
        return [n.stream, n.codes, n.sums, *route, *y]
    return scale, run


@pytest.mark.parametrize("T", [3, 1500])
def test_inputs_of_two_streams_eager_and_captured(T):
    scale, run = joined(T, 256, 16)
    want = [t.clone() for t in run()]
    torch.cuda.synchronize()
    assert not bool(torch.isnan(want[0]).any())
    for _ in range(5):
        got = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for factor in (1.0, -0.5, 1.0):
        scale.fill_(factor)
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        for _ in range(3):
            for t in out:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert rtn.rtn_last_device_status() == 0
