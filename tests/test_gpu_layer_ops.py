"""The layer operators on the GPU against their plain forms in double: types, layouts, odd sizes, strides, refusals."""
import numpy as np
import pytest
import torch

import paper_1912_02057_b200 as rtn
import layer_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ids = lambda v: str(v).replace("torch.", "").replace(" ", "")  # noqa: E731


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


# ---------------------------------------------------------------------------------------------- linear

def linear_case(M, N, K, seed, per_row=True):
    g = np.random.default_rng(seed)
    x, w = (g.choice(np.array([-1, 0, 1], np.int8), size=s, p=[0.3, 0.4, 0.3]) for s in ((M, K), (N, K)))
    na, nw = (M, N) if per_row else (1, 1)
    d = dict(x=x, w=w, a_scale=g.uniform(0.5, 1.5, na).astype(np.float32), a_offset=g.uniform(-0.1, 0.1, na).astype(np.float32),
             w_scale=(g.uniform(0.5, 1.5, nw) / np.sqrt(K)).astype(np.float32),
             w_offset=(g.uniform(-0.1, 0.1, nw) / np.sqrt(K)).astype(np.float32),
             bias=g.normal(size=N).astype(np.float32), residual=g.normal(size=(M, N)).astype(np.float32))
    return d


def packed(d):
    one = torch.tensor([0.5], device="cuda")
    xp, xs = rtn.rtn_ternarize_pack_act(cuda(d["x"]).float(), -one, one)
    wp, ws = rtn.rtn_pack_weights(cuda(d["w"]))
    return (xp, xs, wp, ws[0].contiguous(), d["x"].shape[0], d["w"].shape[0], d["x"].shape[1],
            *(cuda(d[n]) for n in ("a_scale", "a_offset", "w_scale", "w_offset")))


# fp32 roundings: four terms of the affine form (each a product or two and a sum), the bias, the activation (its slope is
# at most 1.13, its own error a few units), the residual
LINEAR_C = 24


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 64, 64), (1, 4096, 4096), (1, 100, 129), (2, 33, 640), (3, 257, 127), (5, 130, 4100),
                                   (8, 1000, 512), (9, 70, 300), (9, 24, 4224), (17, 16, 128), (33, 520, 257), (130, 1000, 512),
                                   (257, 300, 384), (300, 77, 1000), (520, 640, 256), (1100, 528, 130)], ids=ids)
def test_linear_matches_the_plain_form(shape, dtype):
    M, N, K = shape
    for n, (kind, bias, residual, per_row) in enumerate([(0, False, False, True), (1, True, True, False), (2, True, False, True),
                                                         (3, False, True, True), (4, True, True, True)]):
        d = linear_case(M, N, K, 100 + n, per_row)
        r = cuda(d["residual"], dtype) if residual else None
        out = rtn.rtn_ternary_linear(*packed(d), bias=cuda(d["bias"]) if bias else None, activation=kind, residual=r, dtype=dtype)
        want, mag = ref.linear(d["x"], d["w"], d["a_scale"], d["a_offset"], d["w_scale"], d["w_offset"],
                               d["bias"] if bias else None, kind, ref.f64(r) if residual else None)
        assert out.dtype == dtype
        ref.assert_close(out, want, mag, LINEAR_C, f"{shape} act {kind}")
    assert rtn.rtn_last_device_status() == 0


# one launch: tiles of 16, 32, 48 and 64 tokens, a K of its own, and shared by clusters of two, four and eight
@pytest.mark.parametrize("shape", [(16, 6000, 1030), (17, 3000, 2050), (33, 2500, 4224), (33, 16300, 500), (40, 1200, 8200), (50, 3000, 700),
                                   (64, 5000, 130), (63, 900, 4100), (200, 300, 4100), (250, 1000, 1000), (100, 300, 120)], ids=ids)
def test_linear_tiles_and_clusters(shape):
    linear_cases(shape)


# more columns than one round of tiles holds, one row tile and several; several rounds of the largest tiles and a long K
@pytest.mark.parametrize("shape", [(9, 20000, 300), (20, 18900, 300), (64, 20000, 260), (130, 19000, 200), (300, 20000, 130), (3000, 5000, 6000),
                                   (2500, 7001, 1700)], ids=ids)
def test_linear_many_columns_and_many_tiles(shape):
    linear_cases(shape)


def linear_cases(shape):
    M, N, K = shape
    for dtype, kind, bias, residual in ((torch.float32, 2, True, False), (torch.bfloat16, 4, True, True), (torch.float16, 0, False, True)):
        d = linear_case(M, N, K, 100 + kind)
        r = cuda(d["residual"], dtype) if residual else None
        out = rtn.rtn_ternary_linear(*packed(d), bias=cuda(d["bias"]) if bias else None, activation=kind, residual=r, dtype=dtype)
        at = np.linspace(0, M - 1, min(M, 200)).astype(np.int64)              # (rows of the double form)
        want, mag = ref.linear(d["x"][at], d["w"], d["a_scale"][at], d["a_offset"][at], d["w_scale"], d["w_offset"],
                               d["bias"] if bias else None, kind, ref.f64(r)[at] if residual else None)
        ref.assert_close(out[cuda(at)], want, mag, LINEAR_C, f"{shape} {dtype} act {kind}")
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", [(3, 70, 200), (200, 304, 200), (150, 77, 130)], ids=ids)
def test_linear_strided_unaligned_and_in_place(shape, dtype):
    M, N, K = shape
    d = linear_case(M, N, K, 7)
    args = packed(d)
    for offset, stride in ((0, N + 5), (1, N + 3), (0, (N + 63) // 32 * 32)):
        wide = torch.full((M * stride + 8,), 7.0, dtype=dtype, device="cuda")
        out = wide[offset:offset + M * stride].view(M, stride)[:, :N]
        out.copy_(cuda(d["residual"]))
        want, mag = ref.linear(d["x"], d["w"], d["a_scale"], d["a_offset"], d["w_scale"], d["w_offset"], d["bias"], 4, ref.f64(out))
        got = rtn.rtn_ternary_linear(*args, bias=cuda(d["bias"]), activation=rtn.ACT_SILU, residual=out, out=out)
        assert got is out
        ref.assert_close(out, want, mag, LINEAR_C, f"in place, offset {offset}, stride {stride}")
        rest = wide.clone()
        rest[offset:offset + M * stride].view(M, stride)[:, :N] = 7.0
        assert bool((rest == 7.0).all()), "wrote outside its rows"
    # one row of a residual for all rows (stride 0)
    row = cuda(d["residual"][:1], dtype)
    got = rtn.rtn_ternary_linear(*args, residual=row.expand(M, N), dtype=dtype)
    want, mag = ref.linear(d["x"], d["w"], d["a_scale"], d["a_offset"], d["w_scale"], d["w_offset"], None, 0, ref.f64(row))
    ref.assert_close(got, want, mag, LINEAR_C, "broadcast residual")


@pytest.mark.parametrize("shape", [(64, 64, 576), (300, 200, 700), (600, 520, 256)], ids=ids)
def test_linear_without_extras_is_the_gemm(shape):
    d = linear_case(*shape, 3)
    args = packed(d)
    a = rtn.rtn_ternary_linear(*args)
    b = rtn.rtn_ternary_gemm(*args, variant=rtn.VARIANT_I8)
    assert torch.equal(a, b)


def test_linear_special_values_pass_through():
    d = linear_case(4, 40, 64, 5)
    bias = d["bias"].copy()
    bias[:4] = [np.inf, -np.inf, np.nan, 0]
    for M in (4, 40):
        d = linear_case(M, 40, 64, 5)
        for kind in range(5):
            y = rtn.rtn_ternary_linear(*packed(d), bias=cuda(bias), activation=kind).cpu().numpy()
            assert np.all(y[:, 0] == np.inf) and np.isnan(y[:, 2]).all() and np.isfinite(y[:, 3:]).all(), kind
            assert np.all(y[:, 1] == (-np.inf if kind == 0 else 0)) or kind in (2, 3, 4), kind


# ---------------------------------------------------------------------------------------------- norm and rotation

# fp32 roundings: the sum of squares (a tree over at most 64 partial sums of 8 or 16, halved by the root), the root, the quotient, weight
# and rotation
ROTARY_C = 40


def rotary_run(T, Hq, Hk, D, R, layout, norm, dtype, seed=0, positions=True, view=lambda q, k: (q, k), in_place=False):
    g = np.random.default_rng(seed)
    P = 500
    q0, k0 = g.normal(size=(T, Hq, D)) * 2, g.normal(size=(T, max(Hk, 1), D))
    q, k = view(cuda(q0.astype(np.float32), dtype), cuda(k0.astype(np.float32), dtype))
    k = k if Hk else None
    table = rtn.rtn_rotary_table(P, R, 500.0) if R else None
    pos = g.integers(0, P, T) if positions else np.arange(T)
    qw, kw = (g.normal(1, 0.3, D).astype(np.float32), g.normal(1, 0.3, D).astype(np.float32)) if norm else (None, None)
    tab = None if table is None else ref.f64(table)
    wants = [ref.rotary(ref.f64(x), pos, tab, w, 1e-5, layout) if x is not None else None for x, w in ((q, qw), (k, kw))]
    outs = rtn.rtn_qk_norm_rotary(q, k, cuda(pos) if positions else None, table, q_weight=None if qw is None else cuda(qw),
                                  k_weight=None if kw is None or k is None else cuda(kw), eps=1e-5, layout=layout,
                                  out_q=q if in_place else None, out_k=k if in_place else None)
    assert not in_place or (outs[0] is q and outs[1] is k)
    for name, got, want in zip("qk", outs, wants):
        if want is not None:
            ref.assert_close(got, *want, ROTARY_C, name)
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("layout", [rtn.ROTARY_HALF, rtn.ROTARY_INTERLEAVED], ids=["half", "interleaved"])
@pytest.mark.parametrize("dims", [(1, 1, 1, 64, 64), (7, 8, 2, 128, 128), (33, 5, 3, 128, 64), (3, 4, 4, 256, 256), (5, 3, 1, 96, 96),
                                  (4, 2, 2, 80, 48), (6, 3, 2, 50, 50), (2, 2, 1, 7, 6), (3, 2, 0, 128, 32), (2, 1, 1, 1000, 16),
                                  (2500, 32, 8, 128, 128)], ids=ids)
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
def test_norm_and_rotation_match_the_plain_form(dims, layout, norm, dtype):
    rotary_run(*dims, layout, norm, dtype, positions=dims[0] > 3 or dims[0] == 1)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("D", [128, 37])
def test_norm_alone(D, dtype):
    rotary_run(9, 3, 2, D, 0, rtn.ROTARY_HALF, True, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("D,R,extra", [(128, 128, 0), (128, 64, 0), (64, 64, 3), (128, 128, 1)])
@pytest.mark.parametrize("layout", [rtn.ROTARY_HALF, rtn.ROTARY_INTERLEAVED], ids=["half", "interleaved"])
def test_rotation_in_place_on_columns_of_a_projection(D, R, extra, layout, dtype):
    def view(q, k):
        T, Hq, _ = q.shape
        Hk = k.shape[1]
        wide = torch.zeros(T, (Hq + 2 * Hk) * D + extra, dtype=dtype, device="cuda")
        a, b = wide[:, extra:extra + Hq * D].unflatten(1, (Hq, D)), wide[:, extra + Hq * D:extra + (Hq + Hk) * D].unflatten(1, (Hk, D))
        a.copy_(q), b.copy_(k)
        return a, b
    rotary_run(70, 6, 2, D, R, layout, True, dtype, view=view, in_place=True)
    head_major = lambda q, k: (q.transpose(0, 1).contiguous().transpose(0, 1), k.transpose(0, 1).contiguous().transpose(0, 1))  # noqa: E731
    rotary_run(70, 6, 2, D, R, layout, False, dtype, view=head_major, in_place=True)


# (T, Hq, Hk, D, type): one, two and eight heads to a group of lanes, heads of one and of two vectors to a lane
@pytest.mark.parametrize("T,Hq,Hk,D,dtype", [(9, 3, 2, 128, torch.bfloat16), (300, 32, 8, 128, torch.bfloat16), (1000, 33, 7, 128, torch.float16),
                                             (300, 16, 3, 128, torch.float32), (600, 32, 9, 128, torch.float32), (7, 3, 2, 256, torch.float32),
                                             (500, 33, 7, 256, torch.float32), (7, 3, 2, 512, torch.float16), (500, 33, 7, 512, torch.bfloat16)],
                         ids=ids)
@pytest.mark.parametrize("layout", [rtn.ROTARY_HALF, rtn.ROTARY_INTERLEAVED], ids=["half", "interleaved"])
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
@pytest.mark.parametrize("part", [1, 2])
def test_rotation_in_place_of_few_and_many_heads(T, Hq, Hk, D, dtype, layout, norm, part):
    rotary_run(T, Hq, Hk, D, D // part, layout, norm, dtype, in_place=True)
    rotary_run(T, Hq, Hk, D, D // part, layout, norm, dtype)


def test_rotation_keeps_what_lies_past_it():
    """A non-finite value past the rotated part, or in another pair, stays where it is."""
    for layout in (rtn.ROTARY_HALF, rtn.ROTARY_INTERLEAVED):
        for D, R in ((128, 64), (20, 12)):
            q = torch.randn(3, 2, D, device="cuda")
            q[1, 1, R + 1], q[2, 0, R + 2] = float("inf"), float("nan")
            out, _ = rtn.rtn_qk_norm_rotary(q, None, None, rtn.rtn_rotary_table(8, R), layout=layout)
            bad = ~torch.isfinite(out)
            assert bad.sum() == 2 and bool(bad[1, 1, R + 1]) and bool(bad[2, 0, R + 2])


def test_a_position_outside_the_table_is_reported():
    for D, T in ((64, 4), (30, 4)):
        q = torch.ones(T, 2, D, device="cuda")
        table = rtn.rtn_rotary_table(10, D)
        for wrong in (10, -1, 1 << 40):
            pos = torch.tensor([3, wrong, 9, 0], device="cuda")
            out, _ = rtn.rtn_qk_norm_rotary(q, None, pos, table)
            assert torch.isnan(out[1]).all() and torch.isfinite(out[[0, 2, 3]]).all()
            assert rtn.rtn_last_device_status() == 8 and rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("kind", [rtn.ROTARY_SCALE_NONE, rtn.ROTARY_SCALE_LINEAR, rtn.ROTARY_SCALE_BASE, rtn.ROTARY_SCALE_PARTS])
def test_rotary_table(kind):
    R, base, factor, context, low, high, amplitude = 64, 10000.0, 8.0, 4096.0, 1.0, 32.0, 1.2
    rows = 70001
    got = ref.f64(rtn.rtn_rotary_table(rows, R, base, kind, factor, context, low, high, amplitude))
    i = np.arange(R // 2)
    f = base ** (-2.0 * i / R)
    if kind == rtn.ROTARY_SCALE_LINEAR:
        f = f / factor
    if kind == rtn.ROTARY_SCALE_BASE:
        f = (base * factor ** (R / (R - 2))) ** (-2.0 * i / R)
    if kind == rtn.ROTARY_SCALE_PARTS:
        keep = np.clip((context * f / (2 * np.pi) - low) / (high - low), 0, 1)
        f = f * (keep + (1 - keep) / factor)
    angle = np.arange(rows)[:, None] * f
    want = amplitude * np.concatenate([np.cos(angle), np.sin(angle)], 1)
    # angles in double: a few units of 2^-53 times up to 70001 turns of argument, then one rounding to fp32
    assert np.abs(got - want).max() <= amplitude * (2.0 ** -24 + 70001 * 16 * 2.0 ** -53)


# ---------------------------------------------------------------------------------------------- decay attention

def decay_case(lens, H, Hk, Dk, Dv, dtype, seed=0, gap=0, log_decay=None):
    g = np.random.default_rng(seed)
    T = sum(lens)
    make = lambda h, d: cuda(g.normal(size=(T, h, d)).astype(np.float32), dtype)  # noqa: E731
    q, k, v = make(H, Dk), make(Hk, Dk), make(Hk, Dv)
    if log_decay is None:
        log_decay = np.log1p(-np.exp2(-2.0 - 6.0 * np.arange(H) / H)).astype(np.float32)
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return q, k, v, log_decay, start


def decay_check(lens, H, Hk, Dk, Dv, dtype, fresh, seed=0, log_decay=None, scale=None, view=lambda *x: x):
    q, k, v, log_decay, start = decay_case(lens, H, Hk, Dk, Dv, dtype, seed, log_decay=log_decay)
    q, k, v = view(q, k, v)
    g = np.random.default_rng(seed + 1)
    state = None if fresh else g.normal(size=(len(lens), H, Dk, Dv)).astype(np.float32)
    s = Dk ** -0.5 if scale is None else scale
    want, mag, end, mag_end = ref.decay(ref.f64(q), ref.f64(k), ref.f64(v), log_decay, start, state, s)
    out, got = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), max(lens), state=None if fresh else cuda(state), scale=scale)
    c = ref.decay_roundings(log_decay, max(lens), Dk)
    # the tensor-core form rounds scores and states to pairs of bf16 (2^-17 relative) on their way to an output
    ref.assert_close(out, want, mag, c, "out", extra=2.0 ** -15 if dtype == torch.bfloat16 else 0.0)
    ref.assert_close(got, end, mag_end, c, "state")
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("fresh", [True, False], ids=["fresh", "state"])
@pytest.mark.parametrize("lens,H,Hk,Dk,Dv", [
    ([1], 1, 1, 64, 64), ([0, 5, 0], 2, 1, 64, 64), ([127, 1, 128, 129], 2, 2, 64, 64), ([300, 17], 4, 2, 128, 128),
    ([256], 3, 1, 128, 128), ([640], 2, 2, 128, 128), ([65, 2], 2, 1, 128, 64), ([140], 2, 2, 64, 128), ([33, 64], 2, 2, 96, 80),
    ([20], 3, 3, 7, 5), ([40, 3], 2, 1, 256, 256), ([130], 1, 1, 32, 200)], ids=ids)
def test_decay_attention_matches_the_recurrence(lens, H, Hk, Dk, Dv, fresh, dtype):
    decay_check(lens, H, Hk, Dk, Dv, dtype, fresh)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
@pytest.mark.parametrize("D", [64, 128])
def test_one_long_prompt(D, dtype):
    decay_check([5001], 2, 1, D, D, dtype, False)


@pytest.mark.parametrize("value", [0.0, -1e-4, -3.0, -60.0, -400.0, -np.inf])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
def test_decays_from_none_to_all(value, dtype):
    decay_check([200, 31], 2, 2, 64, 64, dtype, False, log_decay=np.array([value, -0.01], np.float32), scale=0.3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
def test_strided_inputs(dtype):
    def columns(q, k, v):
        wide = torch.cat([x.flatten(1) for x in (q, k, v)], 1).contiguous()
        a, b, c = wide.split([x[0].numel() for x in (q, k, v)], 1)
        return a.unflatten(1, q.shape[1:]), b.unflatten(1, k.shape[1:]), c.unflatten(1, v.shape[1:])
    head_major = lambda *x: tuple(t.transpose(0, 1).contiguous().transpose(0, 1) for t in x)  # noqa: E731
    odd = lambda *x: tuple(torch.cat([t.flatten(1), t.flatten(1)[:, :1]], 1)[:, 1:].unflatten(1, t.shape[1:]).copy_(t) for t in x)  # noqa: E731
    for view in (columns, head_major, odd):
        decay_check([150, 70], 4, 2, 64, 64, dtype, False, view=view)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
def test_sequences_do_not_reach_each_other(dtype):
    """NaN and infinities in a neighbour's tokens and state, before and after, change nothing."""
    lens = [70, 60, 200]
    q, k, v, log_decay, start = decay_case(lens, 2, 1, 64, 64, dtype)
    state = torch.randn(3, 2, 64, 64, device="cuda")
    clean = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 200, state=state, state_out=torch.empty_like(state))
    for x in (q, k, v):
        x[:70], x[130:] = float("nan"), float("inf")
    state[0], state[2] = float("nan"), float("inf")
    out, got = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 200, state=state, state_out=torch.empty_like(state))
    assert torch.equal(out[70:130], clean[0][70:130]) and torch.equal(got[1], clean[1][1])


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("D,length,at", [(64, 300, 40), (128, 300, 257), (128, 300, 299), (64, 2500, 1100), (128, 2500, 0), (64, 90, 89)], ids=ids)
def test_a_value_that_is_not_finite_reaches_no_earlier_token(D, length, at, value, dtype):
    q, k, v, log_decay, start = decay_case([length], 2, 2, D, D, dtype)
    run = lambda: rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), length)  # noqa: E731
    clean, end = run()
    keep = v[at, 1, 5].clone()
    v[at, 1, 5] = value                         # one column of one head, from its token on
    out, got = run()
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[at:, 1, 5] = True
    assert torch.equal(out[~bad], clean[~bad]) and not torch.isfinite(out[bad]).any()
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, 1, :, 5] = True
    assert torch.equal(got[~bad], end[~bad]) and not torch.isfinite(got[bad]).any()
    v[at, 1, 5] = keep
    k[at, 1, 7] = value                         # one row of the state: every column of the head
    out, got = run()
    assert torch.equal(out[:, 0], clean[:, 0]) and torch.equal(out[:at], clean[:at]) and not torch.isfinite(out[at:, 1]).any()
    assert torch.equal(got[0, 0], end[0, 0]) and not torch.isfinite(got[0, 1, 7]).any()
    k[at, 1, 7] = 0.5
    clean, end = run()
    q[at, 1, 3] = value                         # one token's output
    out, got = run()
    rest = torch.arange(length, device="cuda") != at
    assert torch.equal(out[rest], clean[rest]) and torch.equal(out[at, 0], clean[at, 0]) and torch.equal(got, end)
    assert not torch.isfinite(out[at, 1]).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
@pytest.mark.parametrize("D", [64, 128])
def test_values_far_from_one_scale_the_result(D, dtype):
    """Every product and sum is linear in v, and a power of two changes no rounding."""
    q, k, v, log_decay, start = decay_case([300, 40], 2, 1, D, D, dtype)
    run = lambda x: rtn.rtn_decay_attention(q, k, x, cuda(log_decay), cuda(start), 300)  # noqa: E731
    out, got = run(v)
    for power in (20, 60):
        big, state = run(v * 2.0 ** power)
        assert torch.equal(big, out * 2.0 ** power) and torch.equal(state, got * 2.0 ** power)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("B,H,Hk,Dk,Dv", [(1, 1, 1, 64, 64), (3, 4, 2, 128, 128), (40, 16, 4, 128, 128), (2, 2, 2, 7, 5), (5, 3, 1, 96, 200),
                                          (2, 2, 1, 256, 256), (300, 2, 2, 64, 64)], ids=ids)
def test_step_matches_the_recurrence(B, H, Hk, Dk, Dv, dtype):
    q, k, v, log_decay, start = decay_case([1] * B, H, Hk, Dk, Dv, dtype)
    g = np.random.default_rng(9)
    pool = B + 3
    slots = g.permutation(pool)[:B].astype(np.int32)
    state = g.normal(size=(pool, H, Dk, Dv)).astype(np.float32)
    want, mag, end, mag_end = ref.decay(ref.f64(q), ref.f64(k), ref.f64(v), log_decay, start, state[slots], Dk ** -0.5)
    c = ref.decay_roundings(log_decay, 1, Dk)
    device = cuda(state)
    out, got = rtn.rtn_decay_attention_step(q, k, v, cuda(log_decay), device, slots=cuda(slots))          # in place
    assert got is device
    ref.assert_close(out, want, mag, c, "out")
    ref.assert_close(got[torch.from_numpy(slots).long().cuda()], end, mag_end, c, "state")
    others = np.setdiff1d(np.arange(pool), slots)
    assert np.array_equal(got.cpu().numpy()[others], state[others])
    # no state yet, states in order
    want, mag, end, mag_end = ref.decay(ref.f64(q), ref.f64(k), ref.f64(v), log_decay, start, None, Dk ** -0.5)
    out, got = rtn.rtn_decay_attention_step(q, k, v, cuda(log_decay), None)
    ref.assert_close(out, want, mag, c, "out, fresh")
    ref.assert_close(got, end, mag_end, c, "state, fresh")
    assert rtn.rtn_last_device_status() == 0


def test_padding_entries_and_bad_slots():
    B, H, D = 4, 2, 64
    for dtype in (torch.float32, torch.bfloat16):
        q, k, v, log_decay, start = decay_case([1] * B, H, H, D, D, dtype)
        state = torch.randn(6, H, D, D, device="cuda")
        keep = state.clone()
        for call in ("step", "prompt"):
            run = (lambda slots, out: rtn.rtn_decay_attention_step(q, k, v, cuda(log_decay), state, slots=slots, out=out)) if call == "step" else \
                (lambda slots, out: rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 1, state=state, slots=slots, out=out))
            state.copy_(keep)
            out = torch.full((B, H, D), 5.0, dtype=dtype, device="cuda")
            run(torch.tensor([2, -1, 5, -7], dtype=torch.int32, device="cuda"), out)
            assert bool((out[[1, 3]] == 0).all()) and bool((out[[0, 2]] != 5).any())
            assert torch.equal(state[[0, 1, 3, 4]], keep[[0, 1, 3, 4]]) and not torch.equal(state[2], keep[2])
            assert rtn.rtn_last_device_status() == 0
            state.copy_(keep)
            run(torch.tensor([2, 6, 0, 1], dtype=torch.int32, device="cuda"), out)
            assert rtn.rtn_last_device_status() == 8
            assert torch.equal(state[[3, 4, 5]], keep[[3, 4, 5]])


def test_bad_sequence_bounds_are_reported_and_skipped():
    for dtype, D in ((torch.float32, 64), (torch.bfloat16, 64), (torch.bfloat16, 128)):
        q, k, v, log_decay, _ = decay_case([100], 2, 2, D, D, dtype)
        for start, longest in (([0, 50, 30], 60), ([0, 50, 120], 80), ([0, 90], 80), ([-3, 40], 80)):
            out, _ = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), torch.tensor(start, dtype=torch.int32, device="cuda"), longest)
            assert rtn.rtn_last_device_status() == 8, (start, longest)
        rtn.rtn_decay_attention(q, k, v, cuda(log_decay), torch.tensor([0, 100], dtype=torch.int32, device="cuda"), 100)
        assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
def test_prompt_then_steps_is_the_longer_prompt(dtype):
    lens, more = [130, 5], 3
    H, Hk, D = 4, 2, 64
    q, k, v, log_decay, start = decay_case([n + more for n in lens], H, Hk, D, D, dtype)
    whole, end = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), max(lens) + more)
    head = torch.cat([torch.arange(s, s + n) for s, n in zip(start, lens)]).cuda()
    first = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    out, state = rtn.rtn_decay_attention(q[head], k[head], v[head], cuda(log_decay), cuda(first), max(lens))
    tol = 2e-2 if dtype == torch.bfloat16 else 1e-4      # two roundings to the type of values of about 10
    assert torch.allclose(out.float(), whole[head].float(), rtol=tol, atol=tol)
    for i in range(more):
        at = torch.tensor([s + n + i for s, n in zip(start, lens)], device="cuda")
        out, state = rtn.rtn_decay_attention_step(q[at], k[at], v[at], cuda(log_decay), state)
        assert torch.allclose(out.float(), whole[at].float(), rtol=tol, atol=tol)
    assert torch.allclose(state, end, rtol=1e-4, atol=1e-3)


def test_state_pool_past_32_bits():
    H, D = 16, 128
    slots_n = (1 << 31) // (H * D * D) + 8                 # element offsets pass 2^31
    pool = torch.empty((slots_n, H, D, D), device="cuda")
    slots = torch.tensor([slots_n - 1, 3, slots_n - 5], dtype=torch.int32, device="cuda")
    pool[slots.long()] = torch.randn(3, H, D, D, device="cuda")
    state = pool[slots.long()].cpu().numpy()
    q, k, v, log_decay, start = decay_case([1] * 3, H, H, D, D, torch.bfloat16)
    want, mag, end, mag_end = ref.decay(ref.f64(q), ref.f64(k), ref.f64(v), log_decay, start, state, D ** -0.5)
    out, _ = rtn.rtn_decay_attention_step(q, k, v, cuda(log_decay), pool, slots=slots)
    c = ref.decay_roundings(log_decay, 1, D)
    ref.assert_close(out, want, mag, c, "step")
    ref.assert_close(pool[slots.long()], end, mag_end, c, "step's state")
    want, mag, end, mag_end = ref.decay(ref.f64(q), ref.f64(k), ref.f64(v), log_decay, start, pool[slots.long()].cpu().numpy(), D ** -0.5)
    out, _ = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 1, state=pool, slots=slots)
    ref.assert_close(out, want, mag, c, "prompt", extra=2.0 ** -15)
    ref.assert_close(pool[slots.long()], end, mag_end, c, "prompt's state")


# ---------------------------------------------------------------------------------------------- all of them

def every_operator():
    """(name, call) of each operator on its own inputs; a call returns its tensors."""
    d = linear_case(5, 256, 256, 1)
    small, args = packed(d), packed(linear_case(300, 256, 256, 2))
    q, k, v, log_decay, start = decay_case([140, 9], 4, 2, 64, 64, torch.bfloat16)
    table, g, s = rtn.rtn_rotary_table(64, 64), cuda(log_decay), cuda(start)
    pos = torch.arange(149, device="cuda") % 64
    w = torch.ones(64, device="cuda")
    state = torch.randn(149, 4, 64, 64, device="cuda")
    new = torch.zeros_like(state)
    return [("linear rows", lambda: [rtn.rtn_ternary_linear(*small, activation=rtn.ACT_GELU, dtype=torch.bfloat16)]),
            ("linear", lambda: [rtn.rtn_ternary_linear(*args, dtype=torch.bfloat16)]),
            ("rotary", lambda: list(rtn.rtn_qk_norm_rotary(q, k, pos, table, w, w))),
            ("prompt", lambda: list(rtn.rtn_decay_attention(q, k, v, g, s, 140))),
            ("step", lambda: list(rtn.rtn_decay_attention_step(q, k, v, g, state, state_out=new)))]


def test_other_streams_and_repeats_give_the_same_bits():
    for name, call in every_operator():
        first = [t.clone() for t in call()]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = call()
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again)), name


def test_graph_capture():
    for name, call in every_operator():
        want = [t.clone() for t in call()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), name


def test_nothing_to_do():
    d = linear_case(1, 64, 64, 1)
    args = list(packed(d))
    args[0], args[1], args[4] = args[0][:0], args[1][:0], 0
    args[7], args[8] = args[7][:0], args[8][:0]
    assert rtn.rtn_ternary_linear(*args, dtype=torch.bfloat16).shape == (0, 64)
    q = torch.empty(0, 2, 64, device="cuda")
    out, _ = rtn.rtn_qk_norm_rotary(q, q, None, rtn.rtn_rotary_table(4, 64))
    assert out.shape == (0, 2, 64)
    g = torch.zeros(2, device="cuda")
    out, state = rtn.rtn_decay_attention(q, q, q, g, torch.zeros(1, dtype=torch.int32, device="cuda"), 0)
    assert out.shape == (0, 2, 64) and state.shape == (0, 2, 64, 64)
    state = torch.randn(3, 2, 64, 64, device="cuda")
    want = state.clone()
    rtn.rtn_decay_attention(q, q, q, g, torch.zeros(4, dtype=torch.int32, device="cuda"), 0, state=state)
    assert torch.equal(state, want)
    rtn.rtn_decay_attention_step(q, q, q, g, state[:0])
    torch.cuda.synchronize()
    assert rtn.rtn_last_device_status() == 0


def test_the_binding_refuses_what_does_not_fit():
    q = torch.zeros(4, 2, 64, device="cuda")
    g, start = torch.zeros(2, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    table = rtn.rtn_rotary_table(8, 64)
    for wrong in (lambda: rtn.rtn_qk_norm_rotary(q.double(), q.double(), None, table),
                  lambda: rtn.rtn_qk_norm_rotary(q, q.half(), None, table),
                  lambda: rtn.rtn_qk_norm_rotary(q, q, torch.zeros(4, dtype=torch.int32, device="cuda"), table),
                  lambda: rtn.rtn_qk_norm_rotary(q.cpu(), None, None, table),
                  lambda: rtn.rtn_qk_norm_rotary(q, None, None, table, q_weight=torch.ones(63, device="cuda")),
                  lambda: rtn.rtn_qk_norm_rotary(q.transpose(1, 2), None, None, table),
                  lambda: rtn.rtn_decay_attention(q, q[:3], q, g, start, 4),
                  lambda: rtn.rtn_decay_attention(q, q, q, g, start.long(), 4),
                  lambda: rtn.rtn_decay_attention(q, q, q, g[:1], start, 4),
                  lambda: rtn.rtn_decay_attention(q, q, q, g, start, 4, state=torch.zeros(1, 2, 64, 64, device="cuda").half()),
                  lambda: rtn.rtn_decay_attention_step(q, q, q, g, torch.zeros(4, 2, 64, 63, device="cuda")),
                  lambda: rtn.rtn_decay_attention_step(q, q, q, g, None, slots=torch.zeros(4, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            wrong()
    for wrong, code in ((lambda: rtn.rtn_qk_norm_rotary(q, None, None, rtn.rtn_rotary_table(8, 66)), 2),
                        (lambda: rtn.rtn_rotary_table(8, 63), 2),
                        (lambda: rtn.rtn_decay_attention(q, q.repeat(1, 2, 1)[:, :3], q.repeat(1, 2, 1)[:, :3], g, start, 4), 2),
                        (lambda: rtn.rtn_decay_attention_step(q, q, q, g, torch.zeros(3, 2, 64, 64, device="cuda")), 2),
                        (lambda: rtn.rtn_qk_norm_rotary(q, q, None, table, q_weight=torch.ones(64, device="cuda")), 1)):
        with pytest.raises(rtn.RtnError) as e:
            wrong()
        assert e.value.code == code
    d = packed(linear_case(4, 64, 64, 1))
    with pytest.raises(ValueError):
        rtn.rtn_ternary_linear(*d, out=torch.empty(4, 63, device="cuda"))
    with pytest.raises(ValueError):
        rtn.rtn_ternary_linear(*d, bias=torch.zeros(63, device="cuda"))
    with pytest.raises(rtn.RtnError):
        rtn.rtn_ternary_linear(*d, activation=9)


# ---------------------------------------------------------------------------------------------- long prompts in segments

@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64), (torch.float16, 128), (torch.float32, 200)],
                         ids=ids)
def test_long_prompts_update_their_states_in_place(dtype, D):
    """Sequences of one and of many segments, states in slots of a pool, read and written in place: the same bits as with states
    of their own, whatever else is in the pool; a padding entry among them."""
    lens, H, Hk = [2100, 3, 900, 130, 0], 2, 1
    q, k, v, log_decay, start = decay_case(lens, H, Hk, D, D, dtype)
    pool = torch.randn(9, H, D, D, generator=torch.Generator().manual_seed(4)).cuda()
    keep = pool.clone()
    slots = torch.tensor([8, 2, 0, -1, 5], dtype=torch.int32, device="cuda")
    live = [0, 1, 2, 4]
    apart = torch.zeros_like(pool)
    out1, _ = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 2100, state=pool, state_out=apart, slots=slots)
    assert torch.equal(pool, keep)
    out2, _ = rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 2100, state=pool, slots=slots)
    at = slots[live].long()
    assert torch.equal(out1, out2) and torch.equal(pool[at], apart[at])
    others = [i for i in range(9) if i not in at.tolist()]
    assert torch.equal(pool[others], keep[others]) and bool((apart[others] == 0).all())
    assert bool((out1[start[3]:start[4]] == 0).all())
    want, mag, end, mag_end = ref.decay(ref.f64(q), ref.f64(k), ref.f64(v), log_decay, start, keep[slots.clamp_min(0).long()].cpu().numpy(), D ** -0.5)
    c = ref.decay_roundings(log_decay, max(lens), D)
    rows = np.r_[0:start[3], start[4]:start[5]]
    ref.assert_close(out1[torch.from_numpy(rows).cuda()], want[rows], mag[rows], c, "out", extra=2.0 ** -15 if dtype == torch.bfloat16 else 0.0)
    ref.assert_close(pool[at], end[live], mag_end[live], c, "state")
    assert rtn.rtn_last_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=ids)
def test_bad_slots_among_long_prompts(dtype):
    lens, H, D = [300, 200, 100], 2, 64
    q, k, v, log_decay, start = decay_case(lens, H, H, D, D, dtype)
    pool = torch.randn(4, H, D, D, device="cuda")
    keep = pool.clone()
    rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 300, state=pool, slots=torch.tensor([1, 4, 3], dtype=torch.int32, device="cuda"))
    assert rtn.rtn_last_device_status() == 8
    assert torch.equal(pool[[0, 2]], keep[[0, 2]]) and not torch.equal(pool[[1, 3]], keep[[1, 3]])


def test_graph_capture_with_scratch():
    """The forms that take scratch memory: a large linear layer, long prompts in segments (both kernels)."""
    calls = []
    args = packed(linear_case(700, 1500, 1024, 2))
    calls.append(lambda: [rtn.rtn_ternary_linear(*args, dtype=torch.bfloat16)])
    for dtype in (torch.bfloat16, torch.float16):
        q, k, v, log_decay, start = decay_case([3000], 2, 1, 64, 64, dtype)
        calls.append(lambda q=q, k=k, v=v, g=cuda(log_decay), s=cuda(start): list(rtn.rtn_decay_attention(q, k, v, g, s, 3000)))
    for call in calls:
        want = [t.clone() for t in call()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for _ in range(2):
            for t in got:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("K", [512, 4096])
def test_a_rows_result_does_not_depend_on_how_many_come_with_it(K):
    """One row, a few (bit planes), some (one launch) and many (two launches): the same bits."""
    d = linear_case(1100, 640, K, 12)
    big = packed(d)
    bias = cuda(d["bias"])
    whole = rtn.rtn_ternary_linear(*big, bias=bias, activation=rtn.ACT_GELU)
    for M in (1, 3, 8, 20, 100, 300, 600):
        part = (big[0][:M], big[1][:M], *big[2:4], M, *big[5:7], big[7][:M], big[8][:M], *big[9:])
        assert torch.equal(rtn.rtn_ternary_linear(*part, bias=bias, activation=rtn.ACT_GELU), whole[:M]), M
    assert rtn.rtn_last_device_status() == 0


# ---------------------------------------------------------------------------------------------- steep decays, values far from one

@pytest.mark.parametrize("log_decay", [-0.3, -0.6, -3.0, -5.0, -8.0, -8.5, -10.0, -20.0])
@pytest.mark.parametrize("dtype,D,longest", [(torch.float32, 64, 70), (torch.float32, 128, 30), (torch.bfloat16, 96, 40), (torch.bfloat16, 64, 15),
                                             (torch.bfloat16, 64, 200)], ids=ids)
@pytest.mark.parametrize("q_power,v_power", [(0, 60), (0, 100), (0, -60), (-60, 60), (60, -60), (-100, 0), (100, 0)])
def test_steep_decays_of_values_far_from_one(log_decay, dtype, D, longest, q_power, v_power):
    """Finite inputs with a finite result give it, whatever the decay: no factor on the way is far from one."""
    lens, H = [longest, 3], 2
    q, k, v, g, start = decay_case(lens, H, 1, D, D, dtype, log_decay=np.array([log_decay, -0.01], np.float32))
    q, v = q * 2.0 ** q_power, v * 2.0 ** v_power
    state = (np.random.default_rng(3).normal(size=(2, H, D, D)) * 2.0 ** v_power).astype(np.float32)
    want, mag, end, mag_end = ref.decay(ref.f64(q), ref.f64(k), ref.f64(v), g, start, state, D ** -0.5)
    out, got = rtn.rtn_decay_attention(q, k, v, cuda(g), cuda(start), longest, state=cuda(state))
    c = ref.decay_roundings(g, longest, D)
    ref.assert_close(out, want, mag, c, "out", extra=2.0 ** -15 if dtype == torch.bfloat16 else 0.0)
    ref.assert_close(got, end, mag_end, c, "state")
    # token by token through the other entry point
    after = cuda(state)
    for t in range(longest):
        rows = [b for b, n in enumerate(lens) if t < n]
        at = start[rows] + t
        slots = torch.tensor(rows, dtype=torch.int32, device="cuda")
        one, _ = rtn.rtn_decay_attention_step(*(x[cuda(at).long()] for x in (q, k, v)), cuda(g), after, slots=slots)
        ref.assert_close(one, want[at], mag[at], c, "token")
    ref.assert_close(after, end, mag_end, c, "tokens' state")


# ---------------------------------------------------------------------------------------------- a stream of the caller's

def calls_that_make_their_results():
    """(name, call(stream)) of every entry point that makes its results."""
    d = linear_case(40, 256, 256, 1)
    x, w = cuda(d["x"]).float(), cuda(d["w"])
    lo, hi = torch.tensor([-0.5], device="cuda"), torch.tensor([0.5], device="cuda")
    args = packed(d)
    four = torch.randint(0, 4, (40, 256), device="cuda").to(torch.uint8)
    fp = rtn.rtn_pack_quaternary(four)
    image = torch.randn(2, 64, 9, 9, device="cuda")
    codes = torch.randint(-1, 2, (64, 64, 3, 3), device="cuda").to(torch.int8)
    cp, cs = rtn.rtn_pack_weights(codes)
    one = torch.ones(1, device="cuda")
    q, k, v, log_decay, start = decay_case([140, 9], 4, 2, 64, 64, torch.bfloat16)
    table, g, s = rtn.rtn_rotary_table(256, 64), cuda(log_decay), cuda(start)
    state = torch.randn(149, 4, 64, 64, device="cuda")
    return [("pack weights", lambda on: rtn.rtn_pack_weights(w, stream=on)),
            ("ternarize", lambda on: rtn.rtn_ternarize_pack_act(x, lo, hi, stream=on)),
            ("gemm", lambda on: [rtn.rtn_ternary_gemm(*args, stream=on)]),
            ("conv", lambda on: [rtn.rtn_ternary_conv2d(image, lo, hi, cp, cs, 64, 3, 3, 1, 1, rtn.PAD_CODE_ZERO, 1.0, 0.0, one, one, stream=on)]),
            ("pack quaternary", lambda on: [rtn.rtn_pack_quaternary(four, stream=on)]),
            ("quaternary gemm", lambda on: [rtn.rtn_quaternary_gemm(fp, fp, 40, 40, 256, stream=on)]),
            ("linear", lambda on: [rtn.rtn_ternary_linear(*args, dtype=torch.bfloat16, stream=on)]),
            ("table", lambda on: [rtn.rtn_rotary_table(300, 64, stream=on)]),
            ("rotary", lambda on: rtn.rtn_qk_norm_rotary(q, k, None, table, stream=on)),
            ("prompt", lambda on: rtn.rtn_decay_attention(q, k, v, g, s, 140, stream=on)),
            ("step", lambda on: rtn.rtn_decay_attention_step(q, k, v, g, None, stream=on))]


def test_results_belong_to_the_stream_that_writes_them():
    """With stream= a result never takes memory whose last use on the current stream is still to come."""
    side = torch.cuda.Stream()
    for name, call in calls_that_make_their_results():
        want = [t.clone() for t in call(None)]
        # tensors of the results' sizes, read late on the current stream and let go of at once
        freed = [torch.full_like(t, 3) for t in want]
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        late = [t.clone() for t in freed]
        del freed
        got = call(side)
        side.synchronize()
        at = {s["address"]: s for s in torch.cuda.memory_snapshot()}
        for t in got:
            segment = next(s for a, s in at.items() if a <= t.data_ptr() < a + s["total_size"])
            assert segment["stream"] == side.cuda_stream, name
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), name
        assert all(bool((t == 3).all()) for t in late), name
    # the default stream, named, from within another one
    default = torch.cuda.default_stream()
    with torch.cuda.stream(side):
        for name, call in calls_that_make_their_results():
            side.synchronize()
            got = call(default)
            default.synchronize()
            want = call(None)
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got)), name
    assert rtn.rtn_last_device_status() == 0


# ---------------------------------------------------------------------------------------------- host threads

@pytest.mark.parametrize("shapes", [((16, 16384, 1024), (64, 16384, 512)), ((1500, 1536, 512), (2000, 4096, 512))], ids=["tiles", "two launches"])
def test_host_threads_with_products_of_different_sizes(shapes):
    """Calls of one kernel with different amounts of shared memory, from several host threads at once: every launch goes through."""
    import threading
    calls, wants = [], []
    for shape in shapes:
        args = packed(linear_case(*shape, 3))
        wants.append(rtn.rtn_ternary_linear(*args))
        calls.append(args)
    torch.cuda.synchronize()
    bad, outs, streams = [], [torch.zeros_like(wants[i % 2]) for i in range(4)], [torch.cuda.Stream() for _ in range(4)]

    def work(i):
        ap, asum, wp, wsum, M, N, K, a_s, a_o, w_s, w_o = calls[i % 2]
        p = [x.data_ptr() for x in (ap, asum, wp, wsum, a_s, a_o, w_s, w_o)]
        f, out, on = rtn.lib().rtn_ternary_linear, outs[i].data_ptr(), streams[i].cuda_stream
        for n in range(1500):
            code = f(p[0], p[1], p[2], p[3], M, N, K, p[4], p[5], M, p[6], p[7], N, None, 0, None, 0, out, N, 0, on)
            if code != 0:
                bad.append(code)
            if n % 100 == 99:
                streams[i].synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad, f"{len(bad)} of 6000 calls refused: {bad[:3]}"
    assert all(torch.equal(outs[i], wants[i % 2]) for i in range(4))
    assert rtn.rtn_last_device_status() == 0


def test_scratch_is_given_back():
    args = packed(linear_case(4096, 4096, 1024, 2))
    q, k, v, log_decay, start = decay_case([3000], 2, 1, 64, 64, torch.bfloat16)
    want, states = rtn.rtn_ternary_linear(*args), rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 3000)
    torch.cuda.synchronize()
    kept = torch.cuda.mem_get_info()[0]
    rtn.rtn_release_scratch()
    assert torch.cuda.mem_get_info()[0] >= kept + 2 * 4096 * 1024              # the expanded operands, a byte per code
    rtn.rtn_release_scratch()
    again, others = rtn.rtn_ternary_linear(*args), rtn.rtn_decay_attention(q, k, v, cuda(log_decay), cuda(start), 3000)
    assert torch.equal(want, again) and all(torch.equal(a, b) for a, b in zip(states, others))
    side = torch.cuda.Stream()
    rtn.rtn_ternary_linear(*args, stream=side)
    rtn.rtn_release_scratch(side)
    assert rtn.rtn_last_device_status() == 0
