"""The work of the operators for layers with 4-bit weights in groups: the linear layer itself, the router to experts,
and the experts' products.

A case is one pass through one of them.  Fields that all cases have: "name", "op" ("linear" | "experts" | "route"),
"T" (tokens) and "dtype" ("float16" | "bfloat16", for the router also "float32").

  linear    K, N       inputs and weight channels
            group      columns that share a scale (0: the whole row)
            zero       integer zero points beside the scales
            glu        the channels are F = N / 2 gates and F values: the output is silu(gate) * value
            bias       with a bias
  experts   the same, and E experts of such weights, top_k slots of a token
            combine    False: a row per (token, slot) out of the token's row, as for gate and value projections
                       True: a row per (token, slot) in, the slots' weighted sum per token out, as for down projections
            pad        tokens at the end of the batch that are padding: their slots have no expert (-1)
  route     E, top_k, score ("softmax" | "sigmoid"), bias, groups, topk_groups, group_top, renormalize, scale
  call      "call"     the public function, output (and workspace) buffers kept by the caller
            "prepared" the same with its arguments marshalled once, as a decode loop keeps it
"""
import math

import torch

own = False

DTYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}


def _linear(name, T, K, N, group, dtype="float16", zero=False, glu=False, bias=False, call="call"):
    return {"name": name, "op": "linear", "T": T, "K": K, "N": N, "group": group, "dtype": dtype, "zero": zero,
            "glu": glu, "bias": bias, "call": call}


def _experts(name, T, E, top_k, K, N, group, dtype="float16", zero=False, glu=False, bias=False, combine=False,
             pad=0, call="call"):
    return {"name": name, "op": "experts", "T": T, "E": E, "top_k": top_k, "K": K, "N": N, "group": group,
            "dtype": dtype, "zero": zero, "glu": glu, "bias": bias, "combine": combine, "pad": pad, "call": call}


def _route(name, T, E, top_k, dtype="float32", score="softmax", bias=False, groups=1, topk_groups=1, group_top=1,
           renormalize=True, scale=1.0, call="call"):
    return {"name": name, "op": "route", "T": T, "E": E, "top_k": top_k, "dtype": dtype, "score": score,
            "bias": bias, "groups": groups, "topk_groups": topk_groups, "group_top": group_top,
            "renormalize": renormalize, "scale": scale, "call": call}


def listed():
    return [
        # the smallest layer of the configurations, one token: launch and host latency only
        _linear("linear_tiny_t1", 1, 512, 512, 128, call="prepared"),
        # one sequence being decoded: the weights pass once
        _linear("linear_decode_13b_qkv_t1", 1, 5120, 15360, 128, zero=True, call="prepared"),
        # sixteen sequences decoded together, gate and up in one call with their product
        _linear("linear_decode_7b_glu_t16", 16, 4096, 22016, 64, dtype="bfloat16", glu=True, call="prepared"),
        # a short prompt of odd length, ragged widths, the smallest groups
        _linear("linear_ragged_t77", 77, 5000, 4090, 32, bias=True),
        # a prompt through the benchmark's layer
        _linear("linear_prompt_7b_up_t2048", 2048, 4096, 11008, 128),
        # the largest layer
        _linear("linear_prompt_70b_up_t4096", 4096, 8192, 28672, 128, dtype="bfloat16", zero=True),
        # one sequence being decoded: gate and up of eight experts, a row each
        _experts("experts_gate_up_t1", 1, 64, 8, 2048, 2816, 128, glu=True, call="prepared"),
        # four sequences: down projections and their weighted sum
        _experts("experts_down_t4", 4, 64, 8, 1408, 2048, 128, dtype="bfloat16", zero=True, combine=True,
                 call="prepared"),
        # a padded batch of short prompts: some thirty rows to an expert, unevenly
        _experts("experts_gate_up_t300", 300, 64, 6, 2048, 2816, 64, dtype="bfloat16", glu=True, pad=13),
        # a long prompt: down projections and their weighted sum
        _experts("experts_down_t2048", 2048, 64, 8, 1408, 2048, 128, combine=True),
        # the router of one sequence being decoded
        _route("route_t1", 1, 64, 8, call="prepared"),
        # the router of a long prompt: balanced by a bias, limited to groups
        _route("route_groups_t4096", 4096, 256, 8, score="sigmoid", bias=True, groups=8, topk_groups=4, group_top=2,
               scale=2.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """linear: T 1 .. 4096, K 512 .. 11008 in steps of 8, N 512 .. 28672 in steps of 2; experts: T 1 .. 2048, 8 .. 128
    experts, 1 .. 8 slots, K 256 .. 4096, N 256 .. 4096; route: T 1 .. 8192, E 8 .. 512.  All over their logarithms,
    and at most the work of the largest listed case."""
    op = rng.choice(("linear", "linear", "experts", "experts", "route"))
    dtype = rng.choice(("float16", "bfloat16"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        E = groups * _log_int(rng, max(2, 8 // groups), 512 // groups)
        topk_groups = rng.randint(1, groups)
        top_k = min(rng.randint(1, 10), topk_groups * (E // groups))
        c = _route("", _log_int(rng, 1, 8192), E, top_k, dtype=rng.choice(("float32", "float16", "bfloat16")),
                   score=rng.choice(("softmax", "sigmoid")), bias=rng.random() < 0.5, groups=groups,
                   topk_groups=topk_groups, group_top=rng.choice((1, 2)), renormalize=rng.random() < 0.7,
                   scale=rng.choice((1.0, 2.5)))
    else:
        common = {"dtype": dtype, "zero": rng.random() < 0.4, "glu": rng.random() < 0.3, "bias": rng.random() < 0.3}
        group = rng.choice((32, 64, 128, 128, 256, 0))
        if op == "linear":
            while True:
                T, K, N = _log_int(rng, 1, 4096), 8 * _log_int(rng, 64, 1376), 2 * _log_int(rng, 256, 14336)
                if T * K * N <= 4096 * 8192 * 28672:
                    break
            c = _linear("", T, K, N, group, **common)
        else:
            E = _log_int(rng, 8, 128)
            T, top_k = _log_int(rng, 1, 2048), rng.randint(1, 8)
            combine = rng.random() < 0.5
            common["glu"] = common["glu"] and not combine
            c = _experts("", T, E, top_k, 8 * _log_int(rng, 32, 512), 2 * _log_int(rng, 128, 2048), group,
                         combine=combine, pad=rng.randint(0, T // 4) if rng.random() < 0.3 else 0, **common)
    if c["T"] <= 64 and rng.random() < 0.5:
        c["call"] = "prepared"
    del c["name"]
    return c


def _groups(case):
    return 1 if case["group"] == 0 else -(-case["K"] // case["group"])


def _ids(case, seed):
    """Distinct experts of every token, some of them more in demand than others; -1 for padding.  (On the host, so that
    `work` knows how many experts take part.)"""
    gen = torch.Generator().manual_seed(77 + int(seed))
    T, E, k = case["T"], case["E"], case["top_k"]
    demand = 0.5 * torch.randn(E, generator=gen)
    noise = -torch.log(-torch.log(torch.rand((T, E), generator=gen).clamp(1e-9, 1 - 1e-7)))
    ids = torch.topk(demand + noise, min(k, E), dim=1).indices.to(torch.int32)
    if k > E:
        ids = torch.cat([ids, ids[:, :1].expand(T, k - E)], dim=1)
    ids[T - case["pad"]:] = -1
    return ids.contiguous()


def _weights(gen, case):
    """Uniform codes, scales U(0.005, 0.02) as of the other forms of the layer, zero points near the middle."""
    lead = (case["E"],) if case["op"] == "experts" else ()
    K, N, G = case["K"], case["N"], _groups(case)
    ld = (K // 2 + 15) // 16 * 16
    return {"w_q": torch.randint(0, 256, lead + (N, ld), generator=gen, device="cuda", dtype=torch.uint8),
            "w_scale": (torch.rand(lead + (N, G), generator=gen, device="cuda") * 0.015 + 0.005).to(torch.float16),
            "w_zero": torch.randint(-3, 4, lead + (N, G), generator=gen, device="cuda", dtype=torch.int8)
            if case["zero"] else None,
            "bias": (torch.randn(lead + (N,), generator=gen, device="cuda") * 0.5).to(DTYPES[case["dtype"]])
            if case["bias"] else None}


def prepare(case, seed):
    """Activations N(0, 1) with some columns ten times as large; router logits N(0, 1.5), as bfloat16 holds them; the
    weights' codes, scales and zero points; for the framework's operators also the weights laid out once and the
    buffers that a serving loop keeps."""
    gen = torch.Generator(device="cuda").manual_seed(20231009 + int(seed))
    dtype = DTYPES[case["dtype"]]
    T = case["T"]
    s = {"case": case}
    if case["op"] == "route":
        logits = torch.randn((T, case["E"]), generator=gen, device="cuda") * 1.5
        s["logits"] = logits.to(torch.bfloat16).to(dtype)
        s["bias"] = torch.randn(case["E"], generator=gen, device="cuda") * 0.05 if case["bias"] else None
        if own:
            s["out"] = (torch.empty((T, case["top_k"]), dtype=torch.int32, device="cuda"),
                        torch.empty((T, case["top_k"]), dtype=torch.float32, device="cuda"))
    else:
        K, N = case["K"], case["N"]
        rows = T * case["top_k"] if case["op"] == "experts" and case["combine"] else T
        x = torch.randn((rows, K), generator=gen, device="cuda")
        x[:, torch.randperm(K, generator=gen, device="cuda")[:max(K // 128, 1)]] *= 10.0
        s["x"] = x.to(dtype)
        s.update(_weights(gen, case))
        if case["op"] == "experts":
            s["ids"] = _ids(case, seed).cuda()
            w = torch.rand((T, case["top_k"]), generator=gen, device="cuda") + 0.1
            s["weights"] = w / w.sum(dim=1, keepdim=True) if case["combine"] else None
        if own:
            from paper_2310_09259_amd import api
            s["w4"] = api.quik_weight_pack_w4g(s["w_q"], s["w_scale"], K, case["group"], w_zero=s["w_zero"],
                                               glu=case["glu"])
            out_rows = T * case["top_k"] if case["op"] == "experts" and not case["combine"] else T
            s["out"] = torch.empty((out_rows, N // 2 if case["glu"] else N), dtype=dtype, device="cuda")
            if case["op"] == "experts":
                s["workspace"] = torch.empty(api.quik_moe_workspace_bytes(T, case["top_k"], s["w4"], case["combine"]),
                                             dtype=torch.uint8, device="cuda")
    if own and case["call"] == "prepared":
        s["call"], _ = _own_call(s, prepared=True)
    return s


def _own_call(s, prepared=False):
    from paper_2310_09259_amd import api
    c = s["case"]
    if c["op"] == "route":
        fn = api.prepare_moe_route if prepared else api.quik_moe_route
        return fn(s["logits"], c["top_k"], bias=s["bias"], score=c["score"], groups=c["groups"],
                  topk_groups=c["topk_groups"], group_top=c["group_top"], renormalize=c["renormalize"],
                  scale=c["scale"], out=s["out"])
    if c["op"] == "linear":
        fn = api.prepare_linear_w4g if prepared else api.quik_linear_w4g
        return fn(s["x"], s["w4"], bias=s["bias"], out=s["out"])
    fn = api.prepare_moe_linear_w4g if prepared else api.quik_moe_linear_w4g
    return fn(s["x"], s["ids"], s["w4"], weights=s["weights"], bias=s["bias"], out=s["out"],
              workspace=s["workspace"])


def _widened(w_q, w_scale, w_zero, K, group):
    """The weights in 32 bits: scale * (code - zero), the codes two to a byte, low nibble first."""
    codes = torch.stack((w_q & 15, w_q >> 4), dim=-1).reshape(w_q.shape[0], -1)[:, :K].to(torch.float32)
    codes = codes - 16.0 * (codes > 7.5)
    g = K if group == 0 else group
    scale = torch.repeat_interleave(w_scale.to(torch.float32), g, dim=1)[:, :K]
    if w_zero is not None:
        codes = codes - torch.repeat_interleave(w_zero.to(torch.float32), g, dim=1)[:, :K]
    return codes * scale


def _product(s, x, e=None):
    """x (32 bits) through one layer's weights, with its bias and, for glu, the product of the halves; in 32 bits."""
    c = s["case"]
    pick = (lambda t: t) if e is None else (lambda t: None if t is None else t[e])
    a = x @ _widened(pick(s["w_q"]), pick(s["w_scale"]), pick(s["w_zero"]), c["K"], c["group"]).t()
    if s["bias"] is not None:
        a = a + pick(s["bias"]).to(torch.float32)
    if c["glu"]:
        gate, value = a[:, :c["N"] // 2], a[:, c["N"] // 2:]
        a = gate / (1.0 + torch.exp(-gate)) * value
    return a


def _plain_experts(s):
    c = s["case"]
    T, k = s["ids"].shape
    flat = s["ids"].reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat + 1, minlength=c["E"] + 1).tolist()
    x = s["x"].to(torch.float32)
    y = torch.zeros((T * k, c["N"] // 2 if c["glu"] else c["N"]), dtype=torch.float32, device="cuda")
    at = counts[0]
    for e, n in enumerate(counts[1:]):
        if n:
            rows = order[at:at + n]
            y[rows] = _product(s, x[rows] if c["combine"] else x[torch.div(rows, k, rounding_mode="floor")], e)
            at += n
    if c["combine"]:
        y = (y.reshape(T, k, -1) * s["weights"][:, :, None]).sum(dim=1)
    return y.to(DTYPES[c["dtype"]])


def _top(values, k):
    """The k largest of every row, largest first, equal ones by index."""
    return torch.sort(values, dim=1, descending=True, stable=True).indices[:, :k]


def _plain_route(s):
    """Scores in 64 bits, since experts next to the border are told apart by them; the weights in 32."""
    c, logits = s["case"], s["logits"].to(torch.float64)
    T, E = logits.shape
    if c["score"] == "softmax":
        score = torch.exp(logits - logits.max(dim=1, keepdim=True).values)
        score = score / score.sum(dim=1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-logits))
    choice = score if s["bias"] is None else score + s["bias"].to(torch.float64)
    if c["groups"] > 1:
        by_group = choice.reshape(T, c["groups"], -1)
        group_score = torch.sort(by_group, dim=2, descending=True).values[:, :, :c["group_top"]].sum(dim=2)
        kept = torch.zeros_like(group_score, dtype=torch.bool)
        kept.scatter_(1, _top(group_score, c["topk_groups"]), True)
        choice = torch.where(kept[:, :, None], by_group, torch.full_like(by_group, -math.inf)).reshape(T, E)
    ids = _top(choice, c["top_k"])
    weights = torch.gather(score, 1, ids).to(torch.float32)
    if c["renormalize"]:
        weights = weights / weights.sum(dim=1, keepdim=True)
    return ids.to(torch.int32), weights * c["scale"]


def run(state):
    """One pass: the layer's output; or the chosen experts and their weights."""
    if own:
        if state["case"]["call"] == "prepared":
            state["call"]()
            return state["out"]
        return _own_call(state)
    op = state["case"]["op"]
    if op == "route":
        return _plain_route(state)
    if op == "experts":
        return _plain_experts(state)
    return _product(state, state["x"].to(torch.float32)).to(DTYPES[state["case"]["dtype"]])


def _weight_bytes(case):
    """One layer's codes, scales, zero points and bias."""
    N, G = case["N"], _groups(case)
    return N * case["K"] // 2 + N * G * (3 if case["zero"] else 2) + (2 * N if case["bias"] else 0)


def work(case):
    """Bytes: activations and the weights that take part read once, outputs written once.  Operations: the products.
    (experts: those of one draw of the routing; others differ by little.)"""
    T = case["T"]
    if case["op"] == "route":
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": T * case["E"] * size + (4 * case["E"] if case["bias"] else 0) + 8 * T * case["top_k"],
                "flops": 4 * T * case["E"]}
    K, N = case["K"], case["N"]
    width = N // 2 if case["glu"] else N
    if case["op"] == "linear":
        return {"bytes": 2 * T * K + _weight_bytes(case) + 2 * T * width, "flops": 2 * T * N * K}
    ids = _ids(case, 0)
    used = torch.unique(ids[ids >= 0]).numel()
    rows, real = T * case["top_k"], T - case["pad"]
    rows_in, rows_out = (real * case["top_k"], T) if case["combine"] else (real, rows)
    return {"bytes": 2 * rows_in * K + used * _weight_bytes(case) + 2 * rows_out * width +
            (8 if case["combine"] else 4) * rows,
            "flops": 2 * real * case["top_k"] * N * K}


def _exact_rows(s, x, lead):
    """float64 product of x with the weights that `lead` selects, column block by column block."""
    c = s["case"]
    q, scale = s["w_q"][lead], s["w_scale"][lead].double()
    zero = s["w_zero"][lead].double() if c["zero"] else None
    g = c["K"] if c["group"] == 0 else c["group"]
    total = torch.zeros((x.shape[0], c["N"]), dtype=torch.float64, device="cuda")
    columns = torch.arange(c["K"], device="cuda")
    step = max(1, (1 << 26) // c["N"])
    for at in range(0, c["K"], step):
        k = columns[at:at + step]
        nibble = torch.bitwise_and(torch.bitwise_right_shift(q[:, k // 2].int(), (4 * (k % 2)).int()), 15)
        code = torch.where(nibble >= 8, nibble - 16, nibble).double()
        if zero is not None:
            code -= zero[:, k // g]
        total += x[:, k].double() @ (code * scale[:, k // g]).t().contiguous()
    if c["bias"]:
        total += s["bias"][lead].double()
    if c["glu"]:
        half = c["N"] // 2
        return total[:, half:] * total[:, :half] / (1 + torch.exp(-total[:, :half]))
    return total


def _exact_route(s):
    c, n = s["case"], s["case"]["E"] // s["case"]["groups"]
    logits = s["logits"].cpu().double().numpy()
    bias = None if s["bias"] is None else s["bias"].cpu().double().numpy()
    ids, weights = [], []
    for row in logits:
        if c["score"] == "softmax":
            peak = float(row.max())
            p = [math.exp(v - peak) for v in row.tolist()]
            total = math.fsum(p)
            p = [v / total for v in p]
        else:
            p = [1.0 / (1.0 + math.exp(-v)) for v in row.tolist()]
        b = p if bias is None else [v + w for v, w in zip(p, bias.tolist())]
        allowed = range(c["groups"])
        if c["groups"] > 1:
            value = [sum(sorted(b[g * n:(g + 1) * n])[::-1][:c["group_top"]]) for g in allowed]
            allowed = sorted(allowed, key=lambda g: (-value[g], g))[:c["topk_groups"]]
        pool = sorted((e for g in allowed for e in range(g * n, (g + 1) * n)), key=lambda e: (-b[e], e))[:c["top_k"]]
        chosen = [p[e] for e in pool]
        norm = math.fsum(chosen) if c["renormalize"] else 1.0
        ids.append(pool)
        weights.append([v / norm * c["scale"] for v in chosen])
    return (torch.tensor(ids, dtype=torch.int32, device="cuda"),
            torch.tensor(weights, dtype=torch.float64, device="cuda"))


def exact(case, seed):
    """What run returns, from the definitions in 64 bits."""
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "route":
        return _exact_route(s)
    if case["op"] == "linear":
        return _exact_rows(s, s["x"], slice(None))
    T, k = s["ids"].shape
    y = torch.zeros((T, k, case["N"] // 2 if case["glu"] else case["N"]), dtype=torch.float64, device="cuda")
    for e in range(case["E"]):
        t, j = torch.nonzero(s["ids"] == e, as_tuple=True)
        if t.numel():
            y[t, j] = _exact_rows(s, s["x"][t * k + j] if case["combine"] else s["x"][t], e)
    if case["combine"]:
        return (y * s["weights"].double()[:, :, None]).sum(dim=1)
    return y.reshape(T * k, -1)
