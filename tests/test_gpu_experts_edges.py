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
