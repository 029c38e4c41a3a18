"""Experts with equal logits at the border of the chosen ones, and others behind them that fp32 scores do not tell from these and
float64 does: against the definition in float64, expert by expert."""
import numpy as np
import pytest

from tests.test_gpu_moe import check_route, route_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("equal", [2, 3, 5])
@pytest.mark.parametrize("top_k", [1, 2, 3])
@pytest.mark.parametrize("at", [5, 9, 70])
def test_a_larger_sigmoid_behind_equal_ones(equal, top_k, at):
    """`equal` logits of 20 in front and one of 25 behind: 1 - 2e-9 and 1 - 1e-11, both 1 in fp32."""
    import torch
    rows = np.full((2, 80), -3.0, np.float32)
    rows[:, :equal] = 20.0
    rows[1, 60:] = -np.inf if at < 60 else 0.5
    rows[:, at] = 25.0
    ids, _ = check_route(torch.from_numpy(rows).cuda(), top_k=top_k, score="sigmoid")
    assert (ids[:, 0] == at).all() and ids[0].tolist() == [at, *range(top_k - 1)]


@pytest.mark.parametrize("bias", [0.0, 1.0])
def test_a_larger_softmax_behind_equal_ones(bias):
    """Two units of 2^-24 apart in the logit: the scores, some 0.1 each, are the same fp32 numbers, or nearly."""
    import torch
    rows = np.full((40, 10), 0.7, np.float32)
    for t in range(40):
        rows[t, 2 + t % 8] += np.float32(2.0 ** -23) * (1 + t // 8)
    for top_k in (1, 2, 9):
        ids, _ = check_route(torch.from_numpy(rows).cuda(), top_k=top_k, bias=np.full(10, bias, np.float32) if bias else None)
        assert ids[:, 0].tolist() == [2 + t % 8 for t in range(40)]


@pytest.mark.parametrize("sigma,shift", [(4.0, 10.0), (8.0, 0.0), (16.0, 10.0), (60.0, -30.0)])
@pytest.mark.parametrize("E,top_k,groups", [(60, 1, 1), (64, 2, 4), (160, 1, 1), (130, 3, 1)])
def test_saturated_scores_of_logits_with_few_bits(E, top_k, groups, sigma, shift):
    """bf16 logits, many of them equal, most sigmoids next to 0 or 1."""
    import torch
    gen = torch.Generator().manual_seed(E + int(sigma))
    rows = (torch.randn((700, E), generator=gen) * sigma + shift).to(torch.bfloat16).float()
    kw = dict(top_k=top_k, score="sigmoid", groups=groups, topk_groups=max(groups // 2, 1), group_top=2 if groups > 1 else 1)
    from paper_2310_09259_amd import api
    ids, _ = api.quik_moe_route(rows.cuda(), **kw)
    ref, _ = route_reference(rows.double().numpy(), **kw)
    assert np.array_equal(ids.cpu().numpy(), ref), np.flatnonzero((ids.cpu().numpy() != ref).any(1))[:5]
