"""Layers of experts: the router (quik_moe_route), the experts' products (quik_moe_linear_w4g) and a whole layer of them,
against their definitions in float64, through the C ABI.  Tolerances of the products as in test_gpu_w4g."""
import math

import numpy as np
import pytest

from tests.test_gpu_w4g import ROUNDS, activations, bounds, check, forced, layer, pack, silu_bounds  # noqa: F401

pytestmark = pytest.mark.gpu


def route_reference(logits, top_k, bias=None, score="softmax", groups=1, topk_groups=1, group_top=1, renormalize=True,
                    scale=1.0):
    """From the definition, expert by expert, in float64 -> ids, weights."""
    T, E = logits.shape
    size = E // groups
    ids, weights = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k))
    for t in range(T):
        l = [float(v) for v in logits[t]]
        on = [not (math.isnan(v) or v == -math.inf) for v in l]
        peak = max((v for v, o in zip(l, on) if o), default=0.0)
        if score == "softmax":
            s = [(1.0 if v == peak else math.exp(v - peak)) if o else 0.0 for v, o in zip(l, on)]
            total = math.fsum(s)
            s = [v / total if total else 0.0 for v in s]
        else:
            s = [(1.0 / (1.0 + math.exp(-v)) if v > -700 else 0.0) if o else 0.0 for v, o in zip(l, on)]
        c = [v + (float(bias[e]) if bias is not None else 0.0) if on[e] else -math.inf for e, v in enumerate(s)]
        c = [-math.inf if math.isnan(v) else v for v in c]
        if groups > 1:
            rank = []
            for g in range(groups):
                best = sorted((v for v in c[g * size:(g + 1) * size] if v > -math.inf), reverse=True)[:group_top]
                if best:
                    rank.append((-sum(best), g))
            kept = {g for _, g in sorted(rank)[:topk_groups]}
            c = [v if e // size in kept else -math.inf for e, v in enumerate(c)]
        chosen = sorted((e for e in range(E) if c[e] > -math.inf), key=lambda e: (-c[e], e))[:top_k]
        total = math.fsum(s[e] for e in chosen) if renormalize else 1.0
        for j, e in enumerate(chosen):
            ids[t, j] = e
            weights[t, j] = (s[e] / total if total else 0.0) * scale
    return ids, weights


def check_route(logits, **kw):
    """ids exactly; weights: fp32 exponentials (2^-21 with their argument's rounding, arguments up to 16 in the tests that
    get weights above 2^-24), sums of up to 1024 scores and two divisions: 2^-18 in all."""
    import torch
    from paper_2310_09259_amd import api
    bias = kw.pop("bias", None)
    b = None if bias is None else torch.from_numpy(bias).cuda()
    ids, weights = api.quik_moe_route(logits, bias=b, **kw)
    ref_ids, ref_w = route_reference(logits.double().cpu().numpy(), bias=bias, **kw)
    assert np.array_equal(ids.cpu().numpy(), ref_ids)
    w = weights.double().cpu().numpy()
    assert np.all(np.abs(w - ref_w) <= 2.0 ** -18 * np.abs(ref_w) + 2.0 ** -40), np.abs(w - ref_w).max()
    return ids, weights


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("T,E,top_k,score,bias,groups,topk_groups,group_top,renormalize,scale", [
    (1, 1, 1, "softmax", False, 1, 1, 1, True, 1.0),
    (3, 2, 2, "sigmoid", True, 1, 1, 1, True, 1.0),
    (1, 64, 8, "softmax", False, 1, 1, 1, True, 1.0),
    (7, 8, 2, "softmax", True, 1, 1, 1, False, 1.0),
    (129, 60, 4, "softmax", False, 1, 1, 1, False, 2.0),
    (65, 65, 6, "sigmoid", True, 1, 1, 1, True, 2.5),
    (33, 160, 6, "softmax", False, 8, 3, 1, False, 16.0),
    (50, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5),
    (9, 96, 32, "sigmoid", False, 3, 2, 5, True, 1.0),
    (5, 1024, 32, "softmax", True, 64, 7, 16, True, 1.0),
    (11, 999, 10, "sigmoid", True, 27, 5, 2, True, 1.0),
    (1030, 12, 3, "softmax", False, 4, 2, 3, True, 1.0),
])
def test_router_against_its_definition(dtype, T, E, top_k, score, bias, groups, topk_groups, group_top, renormalize, scale):
    import torch
    gen = torch.Generator().manual_seed(T * 31 + E)
    buf = torch.full((T, E + 3), float("nan"))
    buf[:, :E] = (torch.randn((T, E), generator=gen) * 2.0).to(torch.bfloat16)   # (equal logits among them)
    logits = buf.to(getattr(torch, dtype)).cuda()[:, :E]
    b = (torch.randn(E, generator=gen) * 0.1).numpy() if bias else None
    check_route(logits, top_k=top_k, bias=b, score=score, groups=groups, topk_groups=topk_groups, group_top=group_top,
                renormalize=renormalize, scale=scale)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_router_choices_next_to_a_border(score):
    """Scores that fp32 cannot tell apart and float64 can, ties, and saturated ones."""
    import torch
    from paper_2310_09259_amd import api
    T, E = 200, 48
    rng = np.random.Generator(np.random.PCG64(4))
    l = rng.standard_normal((T, E)).astype(np.float32)
    l[0::4] = np.float32(0.7)
    l[1::4] = np.float32(0.7) + rng.integers(0, 3, size=(50, E)).astype(np.float32) * np.float32(2 ** -24)
    l[2::4] = 18.0 + rng.integers(0, 40, size=(50, E)).astype(np.float32) * np.float32(0.25)      # sigmoid near 1
    l[3::4] = -110.0 + rng.integers(0, 9, size=(50, E)).astype(np.float32)                       # and near 0
    l[3::4, 5] = 0.0
    for bias in (None, rng.integers(0, 2, size=E).astype(np.float32) * np.float32(2 ** -20)):
        ids, _ = api.quik_moe_route(torch.from_numpy(l).cuda(), 7, score=score,
                                    bias=None if bias is None else torch.from_numpy(bias).cuda())
        ref, _ = route_reference(l.astype(np.float64), 7, bias=bias, score=score)
        assert np.array_equal(ids.cpu().numpy(), ref)


def test_groups_whose_sums_are_small_differences_of_large_choices():
    """Biases of 2^20 and -2^20 in every group: in fp32 the choices are multiples of 2^-3 and 2^-4, and the sums, 1.04 and 1.08,
    come out the other way round."""
    import torch
    scores = [[0.57, 0.47, 0.2, 0.2], [0.55, 0.53, 0.2, 0.2]]
    logits = torch.tensor([math.log(p / (1 - p)) for g in scores for p in g], dtype=torch.float32).reshape(1, 8).cuda()
    bias = np.array([2.0 ** 20, -2.0 ** 20, -2.0 ** 21, -2.0 ** 21] * 2, np.float32)
    ids, _ = check_route(logits, top_k=2, bias=bias, score="sigmoid", groups=2, topk_groups=1, group_top=2)
    assert ids.tolist() == [[4, 5]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_router_masks_that_leave_little_or_nothing(score, groups):
    import torch
    E, inf = 24, float("inf")
    l = torch.randn((9, E), generator=torch.Generator().manual_seed(8))
    l[0] = -inf                                               # nobody
    l[1] = float("nan")
    l[2, 1:] = -inf                                           # one
    l[3, 3:] = float("nan")                                   # three
    l[4, 5] = inf                                             # the limit
    l[5, 5] = inf
    l[5, 9] = inf
    l[6, ::2] = torch.finfo(torch.float32).min                # masks of the type's lowest value
    l[7] = torch.finfo(torch.float32).min
    bias = torch.zeros(E)
    bias[2] = -inf
    bias[7] = float("nan")
    bias[11] = 0.25
    kw = dict(top_k=5, score=score, groups=groups, topk_groups=min(groups, 2), group_top=2 if groups > 1 else 1)
    for b in (None, bias.numpy()):
        ids, weights = check_route(l.cuda(), bias=b, **kw)
        assert (ids[0] == -1).all() and (weights[0] == 0).all() and (ids[1] == -1).all()
        assert bool(torch.isfinite(weights).all())


def moe_reference(x, ids, W, wide, dtype, top_k, glu=False, bias=None, weights=None, rounds=False):
    """-> y, tolerance (float64), rows or weighted sums, of numpy inputs."""
    T = ids.shape[0]
    per_slot = x.shape[0] != T
    width = W.shape[1] // 2 if glu else W.shape[1]
    y, tol = np.zeros((T * top_k, width)), np.zeros((T * top_k, width))
    for r in range(T * top_k):
        e = ids.reshape(-1)[r]
        if 0 <= e < W.shape[0]:
            a, t = bounds(x[None, r if per_slot else r // top_k], W[e], wide[e], dtype, None if bias is None else bias[e], rounds)
            if glu:
                a, t = silu_bounds(a, t)
            y[r], tol[r] = a[0], t[0]
    if weights is None:
        return y, tol
    w = np.where((ids >= 0) & (ids < W.shape[0]), weights, 0.0)[:, :, None]
    y, tol = y.reshape(T, top_k, -1), tol.reshape(T, top_k, -1)
    return (y * w).sum(1), (tol * np.abs(w)).sum(1) + 2.0 ** -23 * top_k * np.abs(y * w).sum(1)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,E,top_k,K,N,group,zero,glu,bias,combine", [
    (1, 4, 1, 128, 32, 128, False, False, False, False),
    (1, 8, 8, 264, 50, 64, True, False, True, True),
    (2, 16, 3, 512, 96, 128, False, True, False, False),
    (3, 2, 2, 136, 34, 32, True, True, True, False),
    (5, 64, 6, 392, 70, 0, True, False, False, True),
    (9, 5, 4, 1024, 48, 256, False, False, True, False),
    (33, 7, 2, 648, 66, 64, True, True, False, True),
    (64, 8, 2, 256, 130, 128, False, False, False, True),
    (100, 3, 3, 136, 18, 32, True, False, True, True),
    (150, 4, 2, 520, 92, 128, True, True, True, False),
    (257, 40, 5, 128, 40, 64, False, False, True, True),
    (400, 2, 1, 264, 300, 128, False, False, False, False),
])
def test_products_against_their_definition(dtype, T, E, top_k, K, N, group, zero, glu, bias, combine):
    """Experts chosen unevenly, some by nobody; the same one twice in a token; ids that are no expert."""
    import torch
    from paper_2310_09259_amd import api
    rng = np.random.Generator(np.random.PCG64(T + E))
    raw = layer(T + K, N, K, group, zero, experts=E)
    w = pack(raw, K, group, glu)
    ids = (E * rng.random((T, top_k)) ** 2).astype(np.int32)
    ids[rng.random((T, top_k)) < 0.1] = -1
    ids[T // 2, 0] = E
    ids[T // 3, -1] = 2 ** 31 - 1
    if T > 2:
        ids[-2] = -1                                          # a token of padding
    weights = rng.uniform(-0.5, 1.0, (T, top_k)).astype(np.float32)
    weights[ids < 0] = np.nan                                 # not looked at
    b = torch.randn((E, N), generator=torch.Generator().manual_seed(5)).to(getattr(torch, dtype)).cuda() if bias else None
    for per_slot in ((True, False) if top_k > 1 else (False,)):
        x = activations(T + N, T * top_k if per_slot else T, K, dtype, ld=K + 8 * (T % 3))
        dead = np.all((ids < 0) | (ids >= E), axis=1)
        if not per_slot:
            x[torch.from_numpy(dead).cuda()] = float("nan")   # padding may hold anything
        y = api.quik_moe_linear_w4g(x, torch.from_numpy(ids).cuda(), w, bias=b,
                                    weights=torch.from_numpy(weights).cuda() if combine else None)
        ref, tol = moe_reference(np.nan_to_num(x.double().cpu().numpy()), ids, raw[3], raw[4], dtype, top_k, glu,
                                 None if b is None else b.double().cpu().numpy(), weights if combine else None)
        check(y, ref, tol, dtype)


def test_a_layer_of_experts_end_to_end_and_as_a_graph():
    """A shared layer and experts with 4-bit weights as a model runs them: router logits from a layer, routing, gates and
    values with their product, down projections with the weighted sum; then the same captured and replayed."""
    import torch
    from paper_2310_09259_amd import api
    E, top_k, K, F = 16, 4, 256, 192
    raw_r, raw_g, raw_d = layer(1, E, K, 128, False), layer(2, 2 * F, K, 64, True, experts=E), layer(4, K, F, 64, False, experts=E)
    router, gate_up, down = pack(raw_r, K, 128), pack(raw_g, K, 64, glu=True), pack(raw_d, F, 64)

    def forward(x):
        ids, weights = api.quik_moe_route(api.quik_linear_w4g(x, router), top_k)
        h = api.quik_moe_linear_w4g(x, ids, gate_up)
        return ids, weights, h, api.quik_moe_linear_w4g(h, ids, down, weights=weights)

    for T in (1, 6, 90):
        x = activations(T, T, K, "bfloat16")
        ids, weights, h, y = forward(x)
        logits = api.quik_linear_w4g(x, router)
        ref_ids, ref_w = route_reference(logits.double().cpu().numpy(), top_k)
        assert np.array_equal(ids.cpu().numpy(), ref_ids)
        ref_h, tol = moe_reference(x.double().cpu().numpy(), ref_ids, raw_g[3], raw_g[4], "bfloat16", top_k, glu=True)
        check(h, ref_h, tol, "bfloat16")
        ref_y, tol = moe_reference(h.double().cpu().numpy(), ref_ids, raw_d[3], raw_d[4], "bfloat16", top_k,
                                   weights=weights.double().cpu().numpy())
        check(y, ref_y, tol, "bfloat16")
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            captured = forward(x)
        for k in range(3):
            x.copy_(activations(T + 50 * k, T, K, "bfloat16"))
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(captured, forward(x)):
                assert torch.equal(a, b), (T, k)


@pytest.mark.parametrize("form", range(13))
@pytest.mark.parametrize("dtype,group,zero,glu,combine", [
    ("float16", 128, True, False, True), ("bfloat16", 64, True, True, False), ("bfloat16", 32, False, False, True),
    ("float16", 32, True, True, True)])
@pytest.mark.parametrize("T,E,top_k", [(4, 16, 3), (90, 5, 2)])
def test_every_kernel_on_every_kind_of_experts(forced, form, dtype, group, zero, glu, combine, T, E, top_k):
    """A row (or token) at a time and by the plan, one expert with most of the rows."""
    import torch
    from paper_2310_09259_amd import api
    K, N = 392, 146
    raw = layer(form, N, K, group, zero, experts=E)
    w = pack(raw, K, group, glu)
    rng = np.random.Generator(np.random.PCG64(form))
    ids = np.where(rng.random((T, top_k)) < 0.7, 2, rng.integers(-1, E + 1, (T, top_k))).astype(np.int32)
    weights = rng.uniform(0.1, 1.0, (T, top_k)).astype(np.float32)
    x = activations(form, T * top_k, K, dtype)
    forced(form)
    y = api.quik_moe_linear_w4g(x, torch.from_numpy(ids).cuda(), w, weights=torch.from_numpy(weights).cuda() if combine else None)
    ref, tol = moe_reference(x.double().cpu().numpy(), ids, raw[3], raw[4], dtype, top_k, glu,
                             weights=weights if combine else None, rounds=form in ROUNDS)
    check(y, ref, tol, dtype)


def test_nobody_is_chosen():
    import torch
    from paper_2310_09259_amd import api
    w = pack(layer(1, 64, 128, 128, True, experts=4), 128, 128)
    for T, top_k in ((1, 2), (40, 3)):
        ids = torch.full((T, top_k), -1, dtype=torch.int32, device="cuda")
        x = torch.full((T, 128), float("nan"), dtype=torch.float16, device="cuda")
        weights = torch.full((T, top_k), float("nan"), device="cuda")
        assert bool((api.quik_moe_linear_w4g(x, ids, w) == 0).all())
        assert bool((api.quik_moe_linear_w4g(x, ids, w, weights=weights) == 0).all())


def test_many_rows_of_one_expert_and_rows_past_the_plans_registers():
    """More rows than the plan keeps between its passes, all but a few of one expert; every row's expert is right."""
    import torch
    from paper_2310_09259_amd import api
    E, K, N, T, top_k = 6, 128, 32, 9001, 3
    raw = layer(5, N, K, 128, False, experts=E)
    w = pack(raw, K, 128)
    rng = np.random.Generator(np.random.PCG64(3))
    ids = np.where(rng.random((T, top_k)) < 0.9, 4, rng.integers(-1, E, (T, top_k))).astype(np.int32)
    x = activations(7, T, K, "bfloat16")
    y = api.quik_moe_linear_w4g(x, torch.from_numpy(ids).cuda(), w)
    xs = x.double().cpu().numpy()
    ref, tol = np.zeros((T * top_k, N)), np.zeros((T * top_k, N))
    for e in range(E):
        r = np.flatnonzero(ids.reshape(-1) == e)
        ref[r], tol[r] = bounds(xs[r // top_k], raw[3][e], raw[4][e], "bfloat16")
    check(y, ref, tol, "bfloat16")


def test_refusals_of_the_binding():
    import torch
    from paper_2310_09259_amd import api
    w = pack(layer(1, 64, 128, 128, True, experts=4), 128, 128)
    dense = pack(layer(1, 64, 128, 128, True), 128, 128)
    x = torch.zeros((3, 128), dtype=torch.float16, device="cuda")
    ids = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    weights = torch.zeros((3, 2), device="cuda")
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    for args, kw, err in (((x, ids, dense), {}, ValueError), ((x, ids.long(), w), {}, TypeError), ((x, ids[0], w), {}, TypeError),
                          ((x, ids.t().contiguous().t(), w), {}, ValueError), ((x[:2], ids, w), {}, ValueError),
                          ((x, ids, w), dict(weights=weights.half()), TypeError), ((x, ids, w), dict(weights=weights[:2]), ValueError),
                          ((x, ids, w), dict(workspace=small), api.QuikError), ((x, ids.cpu(), w), {}, TypeError)):
        with pytest.raises(err):
            api.quik_moe_linear_w4g(*args, **kw)
    with pytest.raises(ValueError):
        api.quik_linear_w4g(x, w)
    logits = torch.zeros((3, 8), device="cuda")
    for kw, err in ((dict(top_k=9), api.QuikError), (dict(top_k=0), api.QuikError), (dict(top_k=2, groups=3), api.QuikError),
                    (dict(top_k=2, bias=torch.zeros(8)), TypeError), (dict(top_k=2, bias=torch.zeros(7, device="cuda")), ValueError),
                    (dict(top_k=2, score="tanh"), ValueError)):
        with pytest.raises(err):
            api.quik_moe_route(logits, **kw)
    with pytest.raises(TypeError):
        api.quik_moe_route(logits.double(), 2)
