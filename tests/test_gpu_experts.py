"""The operators of a layer of routed experts on the GPU against their plain forms in double: types, layouts, odd sizes, masks, refusals."""
import numpy as np
import pytest
import torch

import paper_1912_02057_b200 as rtn
import experts_reference as xref
import layer_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ids = lambda v: str(v).replace("torch.", "").replace(" ", "")  # noqa: E731


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


# ---------------------------------------------------------------------------------------------- routing

# fp32 roundings of a weight: the difference of two logits (at most 30 here, so 30 units of the exponential), the exponential, the sum of up
# to 1024 terms over lanes, registers and a tree, the quotient and the scale
WEIGHT_C = 30 + 4 + 40 + 4


def check_route(x, k, **kw):
    """x: a CUDA tensor of logits."""
    names = dict(score="kind", kept_groups="kept", group_top="top")
    want = xref.route(ref.f64(x), k, **{names.get(n, n): (v.cpu().numpy() if isinstance(v, torch.Tensor) else v) for n, v in kw.items()})
    got = rtn.rtn_route_experts(x, k, **kw)
    assert np.array_equal(got.experts.cpu().numpy(), want[0])
    ref.assert_close(got.weights, want[1], np.abs(want[1]), WEIGHT_C, "weights")
    assert np.array_equal(got.start.cpu().numpy(), want[2])
    assert np.array_equal(got.tokens.cpu().numpy()[:len(want[3])], want[3])
    assert np.array_equal(got.place.cpu().numpy(), want[4])
    return got


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 64, 4), (3, 5, 5), (33, 32, 2), (128, 60, 6), (129, 128, 8), (300, 256, 8), (777, 33, 3),
                                   (70, 1000, 32), (65, 1024, 10), (140, 512, 1)], ids=ids)
def test_route_matches_the_plain_form(shape, dtype):
    T, E, k = shape
    g = np.random.default_rng(T + E)
    x = cuda((1.5 * g.normal(size=(T, E))).astype(np.float32), dtype)
    bias = cuda((0.1 * g.normal(size=E)).astype(np.float32))
    for score in (rtn.SCORE_SOFTMAX, rtn.SCORE_SIGMOID):
        check_route(x, k, score=score)
        check_route(x, k, score=score, bias=bias, renormalise=False, scale=2.5)
    check_route(x, k, renormalise=False)
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("E,groups,kept,top,k", [(64, 8, 4, 2, 8), (64, 8, 1, 1, 8), (60, 4, 3, 2, 6), (256, 8, 4, 2, 8), (96, 32, 5, 3, 7), (30, 3, 2, 10, 4),
                                                 (1024, 16, 3, 2, 9), (33, 11, 2, 1, 3)], ids=ids)
def test_route_in_groups(E, groups, kept, top, k):
    g = np.random.default_rng(E + groups)
    x = cuda((1.5 * g.normal(size=(150, E))).astype(np.float32))
    bias = cuda((0.1 * g.normal(size=E)).astype(np.float32))
    for score in (rtn.SCORE_SOFTMAX, rtn.SCORE_SIGMOID):
        check_route(x, k, score=score, groups=groups, kept_groups=kept, group_top=top)
        check_route(x, k, score=score, bias=bias, groups=groups, kept_groups=kept, group_top=top)


def test_route_ties_go_to_the_lowest_index():
    for T in (3, 200):
        x = torch.zeros(T, 100, device="cuda")
        got = rtn.rtn_route_experts(x, 5)
        assert bool((got.experts == torch.arange(5, device="cuda")).all()) and bool(torch.allclose(got.weights, torch.full_like(got.weights, 0.2)))
        x[:, 50:] = 1.0
        x[:, 60] = -0.0
        check_route(x, 7, bias=torch.zeros(100, device="cuda"), groups=10, kept_groups=3, group_top=2)
        # few different values: many ties
        x = torch.randint(-2, 3, (T, 100), generator=torch.Generator().manual_seed(1)).float().cuda()
        check_route(x, 9)
        check_route(x, 9, bias=x[0].mul(0.25).contiguous(), score=rtn.SCORE_SIGMOID)


def test_route_masked_and_special_logits():
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    rows = [[-inf] * 8, [nan] * 8, [1.0, -inf, nan, 2.0, -inf, -inf, -inf, 0.5], [inf, 0.0, inf, -inf, 1.0, 2.0, nan, 3.0], [low] * 8,
            [low, low, 0.0, low, low, low, low, low], [-300.0, -200.0, -310.0, -250.0, -1000.0, -201.0, -500.0, -400.0],
            [200.0, 300.0, 100.0, 5.0, 90.0, 95.0, 88.0, 120.0]]
    x = torch.tensor(rows, device="cuda")
    for T in (8, 400):
        y = x[torch.arange(T, device="cuda") % 8]
        for score in (rtn.SCORE_SOFTMAX, rtn.SCORE_SIGMOID):
            for kw in (dict(), dict(groups=4, kept_groups=2), dict(renormalise=False)):
                k = 4 if "groups" in kw else 5
                r = rtn.rtn_route_experts(y, k, score=score, **kw)
                want = xref.route(ref.f64(y), k, kind=score, groups=kw.get("groups", 1), kept=kw.get("kept_groups", 1), renormalise=kw.get("renormalise", True))
                assert np.array_equal(r.experts.cpu().numpy(), want[0]), (T, score, kw)
                assert np.array_equal(r.place.cpu().numpy(), want[4]) and np.array_equal(r.start.cpu().numpy(), want[2])
                # differences of logits round at up to 500 units of the exponential
                ref.assert_close(r.weights, want[1], np.abs(want[1]) + 2.0 ** -100, 600, "weights")
    # an expert that the bias takes out, and one that it forces
    bias = torch.zeros(8, device="cuda")
    bias[2], bias[5] = -inf, 100.0
    e = rtn.rtn_route_experts(x[3:4], 3, score=rtn.SCORE_SIGMOID, bias=bias).experts
    assert e[0, 0] == 5 and 2 not in e[0].tolist()


def test_route_choices_near_a_tie_are_those_of_double():
    """Scores plus bias that differ by less than fp32 tells apart."""
    g = np.random.default_rng(5)
    T, E = 256, 64
    x = g.normal(size=(T, E)).astype(np.float32)
    # each row's logits in pairs one unit apart: their sigmoids differ by less than a unit of fp32 for half of them
    x[:, 1::2] = np.nextafter(x[:, 0::2], np.float32(10))
    bias = np.repeat((0.3 * g.normal(size=E // 2)).astype(np.float32), 2)
    check_route(cuda(x), 8, score=rtn.SCORE_SIGMOID, bias=cuda(bias))
    check_route(cuda(x), 8, score=rtn.SCORE_SOFTMAX, bias=cuda(bias), groups=8, kept_groups=3, group_top=2)


def test_route_rows_of_a_wider_tensor_no_tokens_and_no_plan():
    wide = torch.randn(50, 96, device="cuda")
    check_route(wide[:, 7:71], 4)
    check_route(wide[:1].expand(40, 96), 4)
    r = rtn.rtn_route_experts(wide[:0], 4)
    assert r.experts.shape == (0, 4) and bool((r.start == 0).all()) and r.start.numel() == 97
    r, full = rtn.rtn_route_experts(wide, 4, plan=False), rtn.rtn_route_experts(wide, 4)
    assert r.start is None and r.tokens is None and r.place is None and torch.equal(r.experts, full.experts) and torch.equal(r.weights, full.weights)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r = rtn.rtn_route_experts(wide, 4, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(r, full))


@pytest.mark.parametrize("T,E,k,dtype", [(4096, 8, 2, torch.bfloat16), (4133, 100, 8, torch.float16), (5000, 37, 7, torch.float32), (4100, 1024, 8, torch.bfloat16),
                                         (4097, 3, 3, torch.float32), (6000, 132, 1, torch.float32)], ids=ids)
def test_route_of_many_tokens(T, E, k, dtype):
    """Few different values (ties everywhere) and some that are never chosen, rows that begin on and off 16 bytes."""
    g = torch.Generator().manual_seed(T + E)
    x = (torch.randint(-40, 41, (T, E + 3), generator=g).float() / 16)
    x[torch.rand(T, E + 3, generator=g) < 0.05] = -float("inf")
    x[torch.rand(T, E + 3, generator=g) < 0.02] = float("nan")
    x[::97] = -float("inf")
    wide = x.to(dtype).cuda()
    for y in (wide[:, :E].contiguous(), wide[:, 1:E + 1]):
        for score in (rtn.SCORE_SOFTMAX, rtn.SCORE_SIGMOID):
            for renormalise in (True, False):
                r = rtn.rtn_route_experts(y, k, score=score, renormalise=renormalise)
                want = xref.route(ref.f64(y), k, kind=score, renormalise=renormalise)
                for got, exact in zip((r.experts, r.start, r.place), (want[0], want[2], want[4])):
                    assert np.array_equal(got.cpu().numpy(), exact), (score, renormalise)
                rows = int(want[2][-1])
                assert np.array_equal(r.tokens[:rows].cpu().numpy(), want[3][:rows])
                # two exponentials of differences up to 5 (2.5 units each and their argument's rounding), E terms of a sum, a quotient
                ref.assert_close(r.weights, want[1], np.abs(want[1]) + 2.0 ** -100, 40 + E / 2, "weights")


def test_route_refusals():
    x = torch.randn(4, 12, device="cuda")
    for bad in (dict(top_k=0), dict(top_k=33), dict(top_k=2, bias=torch.zeros(11, device="cuda"))):
        with pytest.raises(ValueError):
            rtn.rtn_route_experts(x, **bad)
    for bad in (dict(top_k=13), dict(top_k=2, groups=5), dict(top_k=5, groups=3, kept_groups=1), dict(top_k=2, groups=3, kept_groups=4),
                dict(top_k=2, groups=3, group_top=5), dict(top_k=2, score=2)):
        with pytest.raises(rtn.RtnError):
            rtn.rtn_route_experts(x, **bad)
    with pytest.raises(ValueError):
        rtn.rtn_route_experts(x.double(), 2)
    with pytest.raises(ValueError):
        rtn.rtn_route_experts(x.t(), 2)


# ---------------------------------------------------------------------------------------------- the experts' products

def expert_case(counts, N, K, seed, T=None, per_row=True, wide=1.0):
    """counts: rows of each expert.  T input rows that the rows are gathered from (None: one each, in order)."""
    g = np.random.default_rng(seed)
    E, R = len(counts), int(sum(counts))
    n_in = R if T is None else T
    code = lambda *s: g.choice(np.array([-1, 0, 1], np.int8), size=s, p=[0.3, 0.4, 0.3])  # noqa: E731
    d = dict(x=code(n_in, K), w=code(E, N, K), start=np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), R=R, N=N, K=K,
             tokens=None if T is None else g.integers(0, T, R).astype(np.int32), bias=g.normal(size=(E, N)).astype(np.float32),
             w_scale=(g.uniform(0.5, 1.5, (E, N)) / np.sqrt(K)).astype(np.float32), w_offset=(g.uniform(-0.1, 0.1, (E, N)) / np.sqrt(K)).astype(np.float32),
             a_scale=(g.uniform(0.5, 1.5, n_in) * wide).astype(np.float32), a_offset=g.uniform(-0.1, 0.1, n_in).astype(np.float32))
    if not per_row:
        d["a_scale"], d["a_offset"] = d["a_scale"][:1], d["a_offset"][:1]
    return d


def call_args(d):
    E, N, K = d["w"].shape
    one = torch.tensor([0.5], device="cuda")
    xp, xs = rtn.rtn_ternarize_pack_act(cuda(d["x"]).float(), -one, one)
    wp, ws = rtn.rtn_pack_weights(cuda(d["w"].reshape(E * N, K)))
    return (xp, xs, None if d["tokens"] is None else cuda(d["tokens"]), cuda(d["start"]), wp, ws[0].contiguous(), N, K,
            cuda(d["a_scale"]), cuda(d["a_offset"]), cuda(d["w_scale"].reshape(-1)), cuda(d["w_offset"].reshape(-1)))


def plain(d, bias, kind, gated):
    full = lambda a: np.broadcast_to(a, d["x"].shape[0]) if len(a) == 1 else a  # noqa: E731
    tokens = np.arange(d["R"]) if d["tokens"] is None else d["tokens"]
    return xref.experts(d["x"], tokens, d["start"], d["w"], full(d["a_scale"]), full(d["a_offset"]), d["w_scale"], d["w_offset"],
                        d["bias"] if bias else None, kind, gated)


# fp32 roundings of an output: five of the affine form, the activation's own few units, the product
EXPERTS_C = 24

COUNTS = [[1], [0, 1, 0], [3, 0, 1, 2], [1] * 7, [5, 0, 17, 33, 1], [64, 2], [130, 0, 250, 7], [16] * 12, [300, 1, 0, 0, 515]]


@pytest.mark.parametrize("counts", COUNTS, ids=ids)
@pytest.mark.parametrize("N,K", [(2, 1), (64, 64), (200, 129), (130, 520), (516, 1000)], ids=ids)
def test_experts_match_the_plain_form(counts, N, K):
    for n, (dtype, kind, bias, gated, gather, per_row) in enumerate([
            (torch.float32, 0, False, False, False, True), (torch.bfloat16, 4, True, True, True, True), (torch.float16, 2, True, False, True, False),
            (torch.bfloat16, 3, False, True, False, True), (torch.float32, 1, True, True, True, True)]):
        d = expert_case(counts, N, K, 50 + n, T=max(1, sum(counts) // 2) if gather else None, per_row=per_row)
        args = call_args(d)
        want, mag, live = plain(d, bias, kind, gated)
        b = cuda(d["bias"]) if bias else None
        out = rtn.rtn_ternary_experts(*args, bias=b, activation=kind, gated=gated, dtype=dtype)
        assert out.dtype == dtype and live.all()
        ref.assert_close(out, want, mag, EXPERTS_C, f"{counts} {N}x{K} act {kind}")
        lo, hi = np.float32(-0.2), np.float32(0.3)
        codes, sums = rtn.rtn_ternary_experts(*args, bias=b, activation=kind, gated=gated, t_lo=cuda([lo]), t_hi=cuda([hi]))
        expect = xref.codes_of(want, float(lo), float(hi))
        assert np.array_equal(codes.cpu().numpy(), xref.pack(expect)), f"codes, {counts} {N}x{K} act {kind}"
        assert np.array_equal(sums.cpu().numpy(), expect.sum(1, dtype=np.int32))
    assert rtn.rtn_last_device_status() == 0


def test_experts_long_rows_and_many_experts():
    for counts, N, K in (([2, 30, 0, 3], 66, 8200), ([1, 0, 2] * 100, 40, 300), ([40] * 3, 2050, 256), ([700, 3], 300, 2048), ([0] * 1023 + [9], 10, 130)):
        d = expert_case(counts, N, K, 9, T=50)
        want, mag, _ = plain(d, True, 4, True)
        out = rtn.rtn_ternary_experts(*call_args(d), bias=cuda(d["bias"]), activation=rtn.ACT_SILU, gated=True, dtype=torch.bfloat16)
        ref.assert_close(out, want, mag, EXPERTS_C, f"{N}x{K}")
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("counts", [[2, 0, 3], [40, 9, 0, 200]], ids=ids)
def test_experts_codes_next_to_a_threshold(counts):
    """Thresholds that are outputs, and a unit beside them: the codes are those of the exact values."""
    for gated, kind in ((False, 0), (True, 4), (False, 2)):
        d = expert_case(counts, 256, 300, 31, T=60, wide=3.0)
        want, _, _ = plain(d, True, kind, gated)
        args = call_args(d)
        for i in range(6):
            at = want.flat[(i * 7919) % want.size]
            for hi in (np.float32(abs(at)), np.nextafter(np.float32(abs(at)), np.float32(0))):
                lo = -hi
                codes, sums = rtn.rtn_ternary_experts(*args, bias=cuda(d["bias"]), activation=kind, gated=gated, t_lo=cuda([lo]), t_hi=cuda([hi]))
                expect = xref.codes_of(want, float(lo), float(hi))
                assert np.array_equal(codes.cpu().numpy(), xref.pack(expect))
                assert np.array_equal(sums.cpu().numpy(), expect.sum(1, dtype=np.int32))


@pytest.mark.parametrize("counts", [[2, 0, 3], [40, 9, 0, 200]], ids=ids)
def test_experts_whole_sums_are_exact(counts):
    """Unit scales: the outputs are whole numbers, of both signs and up to K."""
    for K in (1, 127, 700, 4100):
        d = expert_case(counts, 70, K, 8, T=30)
        d["x"][::3], d["w"][0, ::2] = 1, 1
        for n, v in (("a_scale", 1.0), ("a_offset", 0.0), ("w_scale", 1.0), ("w_offset", 0.0)):
            d[n] = np.full_like(d[n], v)
        want, _, _ = plain(d, False, 0, False)
        assert np.array_equal(ref.f64(rtn.rtn_ternary_experts(*call_args(d))), want)


@pytest.mark.parametrize("R,E,N,K", [(20000, 12, 1024, 2048), (30000, 7, 520, 1100), (9000, 60, 2048, 600), (300, 64, 4096, 4096)], ids=ids)
def test_experts_many_tiles_are_exact_every_time(R, E, N, K):
    """Every CTA goes through many tiles, its rings round and round: whole sums against a product in fp32, which is exact, and codes against them; three times."""
    g = torch.Generator(device="cuda").manual_seed(R)
    code = lambda *s: torch.randint(-1, 2, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    x, w = code(R, K), code(E, N, K)
    counts = torch.multinomial(torch.rand(E, generator=g, device="cuda") + 0.2, R, replacement=True, generator=g).bincount(minlength=E)
    start = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    want = torch.cat([x[a:b].float() @ w[e].float().t() for e, (a, b) in enumerate(zip(start[:-1].tolist(), start[1:].tolist()))])
    half, one, zero = (torch.tensor([v], device="cuda") for v in (0.5, 1.0, 0.0))
    xp, xs = rtn.rtn_ternarize_pack_act(x.float(), -half, half)
    wp, ws = rtn.rtn_pack_weights(w.view(E * N, K))
    args = (xp, xs, None, start, wp, ws[0].contiguous(), N, K, one, zero, one, zero)
    t = torch.tensor([20.5], device="cuda")
    gated = want[:, :N // 2] * want[:, N // 2:]
    codes, sums = rtn.rtn_ternarize_pack_act(gated, -t, t)
    for _ in range(3):
        assert torch.equal(rtn.rtn_ternary_experts(*args), want)
        assert torch.equal(rtn.rtn_ternary_experts(*args, gated=True), gated)
        got = rtn.rtn_ternary_experts(*args, gated=True, t_lo=-t, t_hi=t)
        assert torch.equal(got[0], codes) and torch.equal(got[1], sums)
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("counts", [[2, 0, 3, 1], [40, 9, 0, 90]], ids=ids)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_experts_rows_behind_the_last_and_strides(counts, dtype):
    """Rows before the first and behind the last expert's are left as they were, and so is what lies between rows."""
    d = expert_case(counts, 100, 300, 12, T=40)
    R = d["R"]
    d["tokens"] = np.concatenate([np.full(2, -7, np.int32), d["tokens"], np.full(5, 1 << 30, np.int32)])
    want, mag, live = plain({**d, "tokens": d["tokens"][2:2 + R]}, True, 0, False)
    d["start"] = d["start"] + 2
    args = call_args(d)
    for offset, stride in ((0, 100), (1, 103), (0, 128)):
        flat = torch.full(((R + 7) * stride + 8,), 7.0, dtype=dtype, device="cuda")
        out = flat[offset:offset + (R + 7) * stride].view(R + 7, stride)[:, :100]
        got = rtn.rtn_ternary_experts(*args, bias=cuda(d["bias"]), out=out)
        assert got is out
        ref.assert_close(out[2:2 + R], want, mag, EXPERTS_C, f"stride {stride}")
        out[2:2 + R] = 7.0
        assert bool((flat == 7.0).all()), "wrote outside the experts' rows"
    codes, sums = torch.full((R + 7, 32), 9, dtype=torch.uint8, device="cuda"), torch.full((R + 7,), 9, dtype=torch.int32, device="cuda")
    out = torch.full((R + 7, 100), 7.0, dtype=dtype, device="cuda")
    one = torch.tensor([0.25], device="cuda")
    r = rtn.rtn_ternary_experts(*args, bias=cuda(d["bias"]), out=out, t_lo=-one, t_hi=one, out_packed=codes, out_sum=sums)
    assert r[0] is not None and torch.equal(r[0], codes) and r[0].data_ptr() == codes.data_ptr()
    expect = xref.codes_of(want, -0.25, 0.25)
    assert np.array_equal(codes[2:2 + R].cpu().numpy(), xref.pack(expect)) and np.array_equal(sums[2:2 + R].cpu().numpy(), expect.sum(1))
    ref.assert_close(out[2:2 + R], want, mag, EXPERTS_C, "values beside codes")
    for t, v in ((codes, 9), (sums, 9), (out, 7.0)):
        assert bool((t[:2] == v).all()) and bool((t[2 + R:] == v).all())
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("counts", [[2, 1, 3], [50, 3, 60]], ids=ids)
def test_experts_thresholds_of_each_expert(counts):
    d = expert_case(counts, 140, 260, 4)
    want, _, _ = plain(d, False, 4, True)
    lo, hi = np.array([-0.1, -0.5, 0.1], np.float32), np.array([0.1, 0.0, 0.2], np.float32)
    codes, sums = rtn.rtn_ternary_experts(*call_args(d), activation=rtn.ACT_SILU, gated=True, t_lo=cuda(lo), t_hi=cuda(hi))
    of = np.repeat(np.arange(3), counts)
    expect = xref.codes_of(want, lo[of].astype(np.float64)[:, None], hi[of].astype(np.float64)[:, None])
    assert np.array_equal(codes.cpu().numpy(), xref.pack(expect)) and np.array_equal(sums.cpu().numpy(), expect.sum(1))


@pytest.mark.parametrize("counts", [[2, 1, 3], [50, 3, 60]], ids=ids)
def test_experts_special_values(counts):
    d = expert_case(counts, 64, 100, 4)
    d["bias"][:, :3] = [np.inf, -np.inf, np.nan]
    y = rtn.rtn_ternary_experts(*call_args(d), bias=cuda(d["bias"])).cpu().numpy()
    assert np.all(y[:, 0] == np.inf) and np.all(y[:, 1] == -np.inf) and np.isnan(y[:, 2]).all() and np.isfinite(y[:, 3:]).all()
    one = torch.tensor([0.25], device="cuda")
    codes, _ = rtn.rtn_ternary_experts(*call_args(d), bias=cuda(d["bias"]), t_lo=-one, t_hi=one)
    c = codes.cpu().numpy()
    assert np.all(c[:, 0] & 7 == 3) and np.all(c[:, 16] & 7 == 1)            # +1, -1, 0


@pytest.mark.parametrize("counts", [[2, 1, 3], [50, 3, 60]], ids=ids)
def test_experts_indices_out_of_range_are_reported(counts):
    d = expert_case(counts, 64, 100, 4, T=20)
    args = list(call_args(d))
    want, mag, _ = plain(d, False, 0, False)
    one = torch.tensor([0.25], device="cuda")
    bad = args[2].clone()
    bad[1], bad[-1] = 20, -1
    out = rtn.rtn_ternary_experts(*args[:2], bad, *args[3:])
    assert rtn.rtn_last_device_status() == 8 and rtn.rtn_last_device_status() == 0
    assert bool(out[1].isnan().all()) and bool(out[-1].isnan().all())
    ref.assert_close(out[2:-1], want[2:-1], mag[2:-1], EXPERTS_C, "the other rows")
    codes, sums = rtn.rtn_ternary_experts(*args[:2], bad, *args[3:], t_lo=-one, t_hi=one)
    assert not bool(codes[1].any()) and int(sums[1]) == 0 and rtn.rtn_last_device_status() == 8
    # bounds that do not fit: the expert's rows stay, the others' are right
    for start in ([0, counts[0], counts[0] - 1, d["R"]], [0, counts[0], counts[0], d["R"] + 1]):
        out = torch.full((d["R"], 64), 7.0, device="cuda")
        rtn.rtn_ternary_experts(*args[:3], torch.tensor(start, dtype=torch.int32, device="cuda"), *args[4:], out=out)
        assert rtn.rtn_last_device_status() == 8
        own = counts[0] - 1                          # (the row after these is also the third expert's under the first of the two)
        ref.assert_close(out[:own], want[:own], mag[:own], EXPERTS_C, "first expert")


def test_experts_refusals():
    d = expert_case([3, 2], 64, 100, 4, T=4)
    a = list(call_args(d))
    f = rtn.rtn_ternary_experts
    one = torch.tensor([0.25], device="cuda")
    for i, v in ((0, a[0][:-1]), (4, a[4][:-1]), (5, a[5][:-1]), (6, 63), (7, 0), (7, 300), (3, a[3][:1]), (3, a[3].long()), (2, a[2].long()), (8, a[8][:2]),
                 (10, a[10][:5]), (1, a[1].float())):
        with pytest.raises(ValueError):
            f(*a[:i], v, *a[i + 1:])
    with pytest.raises(ValueError):
        f(*a, t_lo=one)
    with pytest.raises(ValueError):
        f(*a, t_lo=-one, t_hi=torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError):
        f(*a, out=torch.empty(5, 63, device="cuda"))
    with pytest.raises(ValueError):
        f(*a, bias=torch.zeros(64, device="cuda"))
    with pytest.raises(rtn.RtnError):
        f(*a, activation=9)
    with pytest.raises(rtn.RtnError):
        f(*a, out=torch.empty(1, 64, device="cuda").expand(5, 64))
    none = a[2][:0]
    assert f(*a[:2], none, torch.zeros(3, dtype=torch.int32, device="cuda"), *a[4:]).shape == (0, 64)


def test_experts_on_other_streams_and_captured():
    """Two graphs of two calls each, replayed in turn on streams of their own, with new inputs: workspaces are not shared."""
    cases = [expert_case([40, 9, 0, 200], 256, 300, 31, T=60), expert_case([3, 1, 2, 0], 256, 300, 32, T=60)]
    args = [call_args(d) for d in cases]
    lo, hi = torch.tensor([-0.2], device="cuda"), torch.tensor([0.3], device="cuda")

    def both(a, s=None):
        c = rtn.rtn_ternary_experts(*a, activation=rtn.ACT_SILU, gated=True, t_lo=lo, t_hi=hi, stream=s)
        return (*c, rtn.rtn_ternary_experts(*a, dtype=torch.bfloat16, stream=s))

    want = [both(a) for a in args]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [both(a, s) for a in args]
    s.synchronize()
    assert all(torch.equal(x, y) for w, g in zip(want, got) for x, y in zip(w, g))
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in args]
    for a in args:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both(a))
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for w, o in zip(want, outs) for x, y in zip(w, o))
    assert rtn.rtn_last_device_status() == 0


# ---------------------------------------------------------------------------------------------- norms around a block

# fp32 roundings of a term: up to 32 of the weighted sum, half of the sum of squares (16 values of a thread and two trees of 5) and the root twice, gate,
# weight, scale and residual
NORM_C = 32 + 2 * 24 + 24


def norm_case(T, W, k, seed, dtype, stream_dtype):
    g = np.random.default_rng(seed)
    R = T * max(k, 1)
    f = lambda *s: g.normal(size=s).astype(np.float32)  # noqa: E731
    place = g.permutation(R).reshape(T, k).astype(np.int32) if k else None
    if k:
        place[g.random((T, k)) < 0.1] = -1
    return dict(branch=cuda(f(R, W), dtype), residual=cuda(f(T, W), stream_dtype), place=None if place is None else cuda(place),
                weights=cuda(g.uniform(0, 1, (T, k)).astype(np.float32)) if k else None, post_weight=cuda(1 + 0.2 * f(W)), gate=cuda(f(T, W), dtype),
                scale=cuda(0.5 + 0.1 * f(W)), norm_weight=cuda(1 + 0.2 * f(W)))


def plain_norm(a, gate_kind=0, eps=1e-6):
    v = {n: None if t is None else t.cpu().numpy() if n == "place" else ref.f64(t) for n, t in a.items()}
    return xref.block_norm(v.get("branch"), v.get("residual"), v.get("place"), v.get("weights"), v.get("post_weight"), v.get("gate"), gate_kind,
                           v.get("scale"), v.get("norm_weight"), eps)


def check_norm(a, gate_kind=0, lo=-0.5, hi=0.4, what=""):
    h, mh, n, mn = plain_norm(a, gate_kind)
    t_lo, t_hi = (torch.tensor([np.float32(t)], device="cuda") for t in (lo, hi))
    r = rtn.rtn_block_norm(a["branch"], **{x: y for x, y in a.items() if x != "branch"}, gate_kind=gate_kind, normed=True, t_lo=t_lo, t_hi=t_hi)
    ref.assert_close(r.stream, h, mh, NORM_C, "stream " + what)
    ref.assert_close(r.normed, n, mn, NORM_C, "normed " + what)
    c = xref.codes_of(n, float(np.float32(lo)), float(np.float32(hi)))
    assert np.array_equal(r.codes.cpu().numpy(), xref.pack(c)), "codes " + what
    assert np.array_equal(r.sums.cpu().numpy(), c.sum(1, dtype=np.int32)), "sums " + what
    s = rtn.rtn_block_norm(a["branch"], **{x: y for x, y in a.items() if x != "branch"}, gate_kind=gate_kind, normed=True)
    assert s.codes is None and torch.equal(s.stream, r.stream) and torch.equal(s.normed, r.normed)
    return r


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", [(1, 1, 0), (2, 8, 2), (5, 31, 0), (3, 64, 4), (4, 129, 1), (3, 1000, 8), (2, 1001, 3), (2, 2048, 4), (3, 4095, 0), (2, 4104, 2),
                                   (2, 5003, 1), (2, 8192, 32), (1, 8200, 2), (1, 16384, 0), (1, 16383, 2)], ids=ids)
def test_block_norm_matches_the_plain_form(shape, dtype):
    T, W, k = shape
    for n, stream_dtype in enumerate(DTYPES):
        a = norm_case(T, W, k, 70 + n, dtype, stream_dtype)
        check_norm(a, n, what="all")
        a["post_weight"] = a["gate"] = None
        check_norm(a, what="one norm")
        a["scale"], a["norm_weight"] = None, None
        check_norm(a, what="sum")
    assert rtn.rtn_last_device_status() == 0


def test_block_norm_parts_left_out():
    a = norm_case(6, 520, 0, 5, torch.bfloat16, torch.float32)
    full = dict(a)
    check_norm({**full, "residual": None}, 2)
    check_norm({"branch": None, "residual": full["residual"], "norm_weight": full["norm_weight"]})
    check_norm({"branch": None, "residual": full["residual"]})
    check_norm({"branch": full["branch"], "scale": full["scale"][:1].contiguous()})
    b = norm_case(6, 520, 3, 6, torch.float16, torch.bfloat16)
    check_norm({**b, "weights": None})
    b["place"][2], b["place"][4, 1:] = -1, -1
    check_norm(b, 1)
    # types where a tensor that decides them is left out
    r = rtn.rtn_block_norm(full["branch"], dtype=torch.float32, normed=True)
    assert r.stream.dtype == torch.float32 and r.normed.dtype == torch.bfloat16
    r = rtn.rtn_block_norm(None, residual=full["residual"], dtype=torch.float16, normed=True)
    assert r.stream.dtype == torch.float32 and r.normed.dtype == torch.float16


@pytest.mark.parametrize("W", [256, 1003], ids=ids)
def test_block_norm_in_place_strided_and_broadcast(W):
    a = norm_case(9, W, 2, 3, torch.bfloat16, torch.float32)
    h, mh, n, mn = plain_norm(a, 1)
    for offset, stride in ((0, W), (0, W + 24), (3, W + 5)):
        flat = torch.full((9 * stride + 16,), 7.0, device="cuda")
        res = flat[offset:offset + 9 * stride].view(9, stride)[:, :W]
        res.copy_(a["residual"])
        wide = torch.full((9, stride + 1), 7.0, device="cuda", dtype=torch.bfloat16)
        r = rtn.rtn_block_norm(**{**a, "residual": res}, gate_kind=1, out=res, normed=wide[:, 1:W + 1])
        assert r.stream.data_ptr() == res.data_ptr()
        ref.assert_close(res, h, mh, NORM_C, "in place")
        ref.assert_close(wide[:, 1:W + 1], n, mn, NORM_C, "strided")
        res.fill_(7.0)
        wide[:, 1:W + 1] = 7.0
        assert bool((flat == 7.0).all()) and bool((wide == 7.0).all()), "wrote outside its rows"
    one = {**a, "gate": a["gate"][:1].expand(9, W), "residual": a["residual"][:1].expand(9, W)}
    check_norm(one, 2, what="one row of a gate and of a residual")


def test_block_norm_codes_next_to_a_threshold():
    """Thresholds that are values, and a unit beside them; terms that cancel."""
    for W, k in ((256, 3), (701, 0)):
        a = norm_case(40, W, k, 21, torch.bfloat16, torch.float32)
        n = plain_norm(a, 2)[2]
        for i in range(6):
            hi = np.float32(abs(n.flat[(i * 7919) % n.size]))
            check_norm(a, 2, lo=-np.nextafter(hi, np.float32(0)), hi=hi, what=f"threshold {i}")
        # a residual that takes most of the branch back: what is left is far below the terms
        a = {"branch": a["branch"][:40], "residual": -a["branch"].float()[:40] * 1.001, "norm_weight": a["norm_weight"]}
        check_norm(a, what="cancelled")


def test_block_norm_thresholds_of_each_value():
    a = norm_case(7, 300, 0, 2, torch.float16, torch.float16)
    n = plain_norm(a, 0)[2]
    g = np.random.default_rng(3)
    lo, hi = g.uniform(-1, 0, 300).astype(np.float32), g.uniform(0, 1, 300).astype(np.float32)
    r = rtn.rtn_block_norm(**a, t_lo=cuda(lo), t_hi=cuda(hi))
    assert np.array_equal(r.codes.cpu().numpy(), xref.pack(xref.codes_of(n, lo.astype(np.float64), hi.astype(np.float64)))) and r.normed is None


def test_block_norm_special_values():
    for W in (256, 131):
        x = torch.randn(4, W, device="cuda")
        x[0, 5], x[1, 6], x[2] = float("nan"), float("inf"), 0.0
        w = torch.ones(W, device="cuda")
        one = torch.tensor([0.25], device="cuda")
        r = rtn.rtn_block_norm(None, residual=x, norm_weight=w, normed=True, t_lo=-one, t_hi=one)
        assert bool(r.normed[0].isnan().all()) and not bool(r.codes[0].any()) and int(r.sums[0]) == 0
        assert bool((r.normed[1][:6] == 0).all()) and bool(r.normed[1][6].isnan())
        assert bool((r.normed[2] == 0).all()) and not bool(r.codes[2].any()) and bool(r.normed[3].isfinite().all())
        # squares beyond fp32: the codes are the exact values' all the same
        big = torch.randn(2, W, device="cuda") * 1e25
        c = xref.codes_of(plain_norm({"branch": None, "residual": big, "norm_weight": w})[2], -0.25, 0.25)
        r = rtn.rtn_block_norm(None, residual=big, norm_weight=w, t_lo=-one, t_hi=one)
        assert np.array_equal(r.codes.cpu().numpy(), xref.pack(c))


def test_block_norm_places_out_of_range_are_reported():
    a = norm_case(5, 200, 2, 2, torch.bfloat16, torch.float32)
    h, mh, _, _ = plain_norm({**a, "place": a["place"].clone()}, 0)
    a["place"][3, 1] = 10
    one = torch.tensor([0.25], device="cuda")
    r = rtn.rtn_block_norm(**a, t_lo=-one, t_hi=one)
    assert rtn.rtn_last_device_status() == 8 and rtn.rtn_last_device_status() == 0
    assert bool(r.stream[3].isnan().all()) and not bool(r.codes[3].any())
    keep = [0, 1, 2, 4]
    ref.assert_close(r.stream[keep], h[keep], mh[keep], NORM_C, "the other rows")


def test_block_norm_refusals():
    a = norm_case(5, 200, 2, 2, torch.bfloat16, torch.float32)
    f = rtn.rtn_block_norm
    one = torch.tensor([0.25], device="cuda")
    for bad in (dict(weights=a["weights"][:4]), dict(place=a["place"].long()), dict(gate=a["gate"].float()), dict(residual=a["residual"][:, :100]),
                dict(scale=torch.ones(3, device="cuda")), dict(norm_weight=torch.ones(100, device="cuda")), dict(t_lo=one), dict(out=torch.empty(5, 200)),
                dict(normed=torch.empty(5, 200, device="cuda")), dict(branch=None, residual=None), dict(out_sum=torch.empty(5, device="cuda").int())):
        with pytest.raises(ValueError):
            f(**{**a, **bad})
    for bad in (dict(gate_kind=3), dict(eps=-1.0), dict(branch=None, place=None, weights=None), dict(place=None)):
        with pytest.raises((rtn.RtnError, ValueError)):
            f(**{**a, **bad})
    with pytest.raises(rtn.RtnError):
        f(torch.zeros(2, 16385, device="cuda"))
    with pytest.raises(rtn.RtnError):
        f(None, residual=a["residual"], out=torch.empty(1, 200, device="cuda").expand(5, 200))
    assert f(a["branch"][:0]).stream.shape == (0, 200)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    want, got = f(**a), f(**a, stream=s)
    s.synchronize()
    assert torch.equal(want.stream, got.stream)


@pytest.mark.parametrize("W", [136, 1003], ids=ids)
def test_block_norm_infinite_parameters_stay_in_their_column(W):
    """What the first column is multiplied with reaches no other one, whatever stands behind the row's end."""
    a = norm_case(3, W, 0, 4, torch.float32, torch.float32)
    a["scale"][0] = float("inf")
    a["norm_weight"] = None
    r = rtn.rtn_block_norm(**a)
    assert bool(r.stream[:, 0].isinf().all()) and bool(r.stream[:, 1:].isfinite().all())
    a["norm_weight"] = torch.ones(W, device="cuda")
    n = rtn.rtn_block_norm(**a, normed=True).normed
    assert bool(n[:, 0].isnan().all()) and bool((n[:, 1:] == 0).all())


def test_route_many_tokens():
    """More blocks than one launch adds up, tokens of a block up to the most, and the choices of a few rows."""
    T, E, k = 80000, 32, 2
    x = torch.randn(T, E, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    x[::7, :3] = float("-inf")
    r = rtn.rtn_route_experts(x, k)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(r.experts.long(), order)
    flat = order.flatten()
    at = torch.sort(flat, stable=True).indices
    assert torch.equal(r.tokens.long(), at // k) and torch.equal(r.place.flatten()[at].long(), torch.arange(T * k, device="cuda"))
    assert torch.equal(r.start[1:].long(), torch.bincount(flat, minlength=E).cumsum(0)) and int(r.start[0]) == 0
    for T in (16, 17, 4000, 10000, 40000):
        s = rtn.rtn_route_experts(x[:T], k)
        assert torch.equal(s.experts, r.experts[:T]) and torch.equal(s.start[1:].long(), torch.bincount(flat[:T * k], minlength=E).cumsum(0))
        at = torch.sort(flat[:T * k], stable=True).indices
        assert torch.equal(s.tokens.long(), at // k)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("E,k", [(64, 8), (60, 3), (129, 8), (7, 7), (256, 1)], ids=ids)
def test_route_is_the_same_for_a_token_among_many(E, k, dtype):
    """Special logits among them; rows on every alignment."""
    T = 5000
    g = torch.Generator(device="cuda").manual_seed(E)
    x = (2 * torch.randn(T, E, generator=g, device="cuda")).to(dtype)
    x[torch.rand(T, E, generator=g, device="cuda") < 0.02] = float("-inf")
    x[torch.rand(T, E, generator=g, device="cuda") < 0.01] = float("nan")
    x[torch.rand(T, E, generator=g, device="cuda") < 0.01] = float("inf")
    x[torch.rand(T, E, generator=g, device="cuda") < 0.05] = torch.finfo(dtype).max
    x[5], x[6, 1:], x[7] = float("-inf"), float("nan"), torch.finfo(dtype).min
    x[8:40] = x[8:40].round()
    for kw in (dict(), dict(score=rtn.SCORE_SIGMOID), dict(renormalise=False, scale=0.5), dict(score=rtn.SCORE_SIGMOID, renormalise=False)):
        many = rtn.rtn_route_experts(x, k, **kw)
        for a in (0, 4000):
            few = rtn.rtn_route_experts(x[a:a + 700], k, **kw)
            assert torch.equal(few.experts, many.experts[a:a + 700])
            # (a softmax's sum over all experts goes in another order)
            assert torch.allclose(few.weights, many.weights[a:a + 700], rtol=WEIGHT_C * 2.0 ** -23, atol=1e-37)
        flat = many.experts.flatten().long()
        assert torch.equal(many.start[1:].long(), torch.bincount(flat[flat >= 0], minlength=E).cumsum(0))
