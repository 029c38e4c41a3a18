"""Layers with 4-bit weights in groups (quik_linear_w4g) against the definition in float64, through the C ABI.

Tolerance, per output, with u = half a step of the output's type (fp16 2^-11, bf16 2^-8): the output is rounded once, u |y|;
where the kernel rounds the weights to that type first (ROUNDS), each product is off by u |x w| at most; the fp32 sums add
2^-24 of the absolute products per term, at most K terms deep (bf16 widens codes by an offset of 128, which makes products up
to (136 + |q - z|) / |q - z| larger: its share is counted on 144 |x| s).  Nothing else is rounded."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

STEP = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}      # half a step of the smallest numbers


ROUNDS = (9, 10)                 # kernels (quik_debug_w4g_form) that may round the weights


@pytest.fixture
def forced():
    """Sets the kernel of w4g products; automatic again afterwards."""
    from paper_2310_09259_amd import api
    yield api.quik_debug_set_w4g_form
    api.quik_debug_set_w4g_form(-1)


def layer(seed, N, K, group, zero, experts=0, pad=16):
    """Raw weights (numpy) and their matrix in float64, [experts,] N, K."""
    rng = np.random.Generator(np.random.PCG64(seed))
    lead = (experts,) if experts else ()
    G = 1 if group == 0 else -(-K // group)
    ldw = (K // 2 + 15) // 16 * 16 + (pad if seed % 2 else 0)
    codes = rng.integers(-8, 8, size=(*lead, N, K))
    w_q = rng.integers(0, 256, size=(*lead, N, ldw), dtype=np.uint8)
    w_q[..., :K // 2] = (codes[..., 0::2] & 15) | ((codes[..., 1::2] & 15) << 4)
    scale = rng.uniform(0.005, 0.02, size=(*lead, N, G)).astype(np.float16)
    scale[..., 0, :] = 0                                     # a channel without weight
    z = rng.integers(-8, 9, size=(*lead, N, G)).astype(np.int8) if zero else None
    of = np.arange(K) // (group or K)
    q = codes - (z.astype(np.int64)[..., of] if zero else 0)
    return w_q, scale, z, q * scale.astype(np.float64)[..., of], np.abs(q) + 136.0


def pack(raw, K, group, glu=False):
    import torch
    from paper_2310_09259_amd import api
    w_q, scale, z = (None if v is None else torch.from_numpy(v).cuda() for v in raw[:3])
    return api.quik_weight_pack_w4g(w_q, scale, K, group, w_zero=z, glu=glu)


def activations(seed, T, K, dtype, ld=None):
    import torch
    gen = torch.Generator().manual_seed(seed)
    buf = torch.full((T, ld or K), float("nan"), dtype=getattr(torch, dtype))
    buf[:, :K] = torch.randn((T, K), generator=gen).to(buf.dtype)
    return buf.cuda()[:, :K]


def bounds(x, W, wide, dtype, bias=None, rounds=False):
    """a (float64) and the tolerance of a before its final rounding; wide: |q - z| + 136 for every weight."""
    a = x @ W.T
    mag = np.abs(x) @ np.abs(W).T
    # |W| / |q - z| = the scale: sums of bf16 run on products of up to (|q - z| + 136) |x| s
    s = np.divide(np.abs(W), wide - 136.0, out=np.zeros_like(W), where=wide > 136.0)
    run = np.abs(x) @ (np.maximum(np.abs(W), s * wide) if dtype == "bfloat16" else np.abs(W)).T
    tol = (STEP[dtype] * mag if rounds else 0.0) + 2.0 ** -24 * (x.shape[1] + 8) * run
    if bias is not None:
        a = a + bias
        tol = tol + 2.0 ** -23 * np.abs(a)
    return a, tol


def silu_bounds(a, tol):
    """silu(gate) * value and its tolerance: |d silu| <= 1.1 |d gate|; the exponential and the reciprocal of the kernel
    are good to 2^-19 of the result up to |gate| = 88 (2^-22 each, the exponential's argument rounded)."""
    h = a.shape[1] // 2
    g, v, tg, tv = a[:, :h], a[:, h:], tol[:, :h], tol[:, h:]
    s = g / (1.0 + np.exp(-np.clip(g, -700, 700)))
    return s * v, 1.1 * tg * (np.abs(v) + tv) + np.abs(s) * tv + 2.0 ** -19 * np.abs(s * v)


def check(y, ref, tol, dtype):
    y = y.double().cpu().numpy()
    limit = STEP[dtype] * (np.abs(ref) + tol) + tol + TINY[dtype]
    err = np.abs(y - ref)
    assert np.all(err <= limit), (float(np.nanmax(err / limit)), np.argwhere(~(err <= limit))[:5].tolist())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,K,N,group,zero,glu,bias", [
    (1, 512, 512, 128, False, False, False),
    (1, 8, 1, 32, True, False, True),            # the smallest
    (1, 136, 17, 128, True, False, False),       # a last group of eight columns, a channel more than a block
    (2, 1000, 62, 32, True, True, True),         # halves of 31 channels
    (5, 4096, 96, 0, False, False, False),       # one group for the row
    (15, 1416, 130, 256, True, False, True),
    (16, 640, 2, 64, False, True, False),        # one gate, one value
    (17, 264, 50, 64, True, False, False),
    (31, 2048, 48, 128, False, True, True),
    (33, 520, 34, 32, False, False, True),
    (64, 1024, 100, 128, True, True, False),
    (65, 776, 66, 64, True, False, True),
    (100, 5000, 40, 32, False, False, False),
    (129, 384, 258, 128, True, True, True),
    (256, 256, 256, 128, False, False, False),
    (300, 904, 514, 64, True, False, True),
    (515, 1160, 90, 0, True, True, False),
    (1030, 128, 516, 32, False, False, True),
])
def test_layer_against_its_definition(dtype, T, K, N, group, zero, glu, bias):
    import torch
    from paper_2310_09259_amd import api
    raw = layer(T * 7 + K, N, K, group, zero)
    w = pack(raw, K, group, glu)
    x = activations(T + N, T, K, dtype, ld=K + 8 * (T % 3))
    b = torch.randn(N, generator=torch.Generator().manual_seed(5)).to(x.dtype).cuda() if bias else None
    y = api.quik_linear_w4g(x, w, bias=b)
    a, tol = bounds(x.double().cpu().numpy(), raw[3], raw[4], dtype, None if b is None else b.double().cpu().numpy(),
                    rounds=api.quik_debug_w4g_form(T, N, K, glu) in ROUNDS)
    if glu:
        a, tol = silu_bounds(a, tol)
    check(y, a, tol, dtype)


def test_output_with_gaps_leaves_the_rest_alone_and_rows_do_not_mix():
    import torch
    from paper_2310_09259_amd import api
    for T in (3, 70, 300):
        K, N = 392, 77
        raw = layer(T, N, K, 64, True)
        w = pack(raw, K, 64)
        x = activations(T, T, K, "float16", ld=400)
        x[1] = float("nan")                                  # a row without meaning stays one
        buf = torch.full((T, N + 6), 7.0, dtype=torch.float16, device="cuda")
        api.quik_linear_w4g(x, w, out=buf[:, 3:3 + N])
        keep = [t for t in range(T) if t != 1]
        a, tol = bounds(x[keep].double().cpu().numpy(), raw[3], raw[4], "float16")
        check(buf[keep, 3:3 + N], a, tol, "float16")
        assert bool((buf[:, :3] == 7).all()) and bool((buf[:, 3 + N:] == 7).all())


def test_prepared_call_and_graph_replay_give_the_same_bits():
    import torch
    from paper_2310_09259_amd import api
    for T in (1, 40, 200):
        K, N = 512, 320
        w = pack(layer(3, N, K, 128, True), K, 128, glu=True)
        x = activations(9, T, K, "bfloat16")
        first = api.quik_linear_w4g(x, w).clone()
        call, y = api.prepare_linear_w4g(x, w)
        call()
        assert torch.equal(y, first)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            z = api.quik_linear_w4g(x, w)
        other = activations(10, T, K, "bfloat16")
        for k in range(4):
            x.copy_(other if k % 2 else activations(9, T, K, "bfloat16"))
            z.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(z, api.quik_linear_w4g(x, w)), k
            assert torch.equal(z, first) == (k % 2 == 0)


@pytest.mark.parametrize("form", range(13))
@pytest.mark.parametrize("dtype,group,zero,glu,bias", [
    ("float16", 128, True, False, True), ("bfloat16", 64, False, False, False), ("float16", 32, True, True, False),
    ("bfloat16", 128, True, True, True), ("bfloat16", 32, True, False, False), ("float16", 64, False, True, True)])
@pytest.mark.parametrize("T,K,N", [(3, 904, 146), (70, 392, 530), (275, 1288, 300)])
def test_every_kernel_on_every_kind_of_layer(forced, form, dtype, group, zero, glu, bias, T, K, N):
    """Odd numbers of tiles of columns, so that groups that split K end differently; ragged rows and channels."""
    import torch
    from paper_2310_09259_amd import api
    raw = layer(form + T, N, K, group, zero)
    w = pack(raw, K, group, glu)
    x = activations(T + form, T, K, dtype)
    b = torch.randn(N, generator=torch.Generator().manual_seed(6)).to(x.dtype).cuda() if bias else None
    forced(form)
    y = api.quik_linear_w4g(x, w, bias=b)
    a, tol = bounds(x.double().cpu().numpy(), raw[3], raw[4], dtype, None if b is None else b.double().cpu().numpy(),
                    rounds=form in ROUNDS)
    if glu:
        a, tol = silu_bounds(a, tol)
    check(y, a, tol, dtype)


def test_rows_far_into_a_matrix_of_more_than_4_gb(forced):
    import torch
    from paper_2310_09259_amd import api
    T, ld, K, N = 70003, 32768, 256, 48                     # rows 64 KB apart: 4.6 GB
    x = torch.empty((T, ld), dtype=torch.float16, device="cuda")[:, :K]
    x.copy_(torch.randn((T, K), generator=torch.Generator().manual_seed(1)).half())
    raw = layer(11, N, K, 128, True)
    w = pack(raw, K, 128)
    at = torch.tensor([0, 1, 40000, 65535, 65536, 65537, T - 2, T - 1])
    a, tol = bounds(x[at.cuda()].double().cpu().numpy(), raw[3], raw[4], "float16", rounds=True)
    for form in (-1, 5, 10):
        forced(form)
        check(api.quik_linear_w4g(x, w)[at.cuda()], a, tol, "float16")


def test_other_stream_and_refusals_of_the_binding():
    import torch
    from paper_2310_09259_amd import api
    raw = layer(2, 96, 256, 64, True)
    w = pack(raw, 256, 64)
    x = activations(1, 20, 256, "float16")
    y = api.quik_linear_w4g(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = api.quik_linear_w4g(x, w)
        call, p = api.prepare_linear_w4g(x, w)
    call()                                                  # on the stream it was prepared on
    side.synchronize()
    assert torch.equal(y, z) and torch.equal(y, p)
    one = api.quik_linear_w4g(x[:1].t().contiguous().t(), w)   # one row, whatever its stride
    assert torch.equal(one, y[:1])
    for bad, err in ((x.float(), TypeError), (x[:, :248], ValueError), (x.t().contiguous().t(), ValueError), (x[0], ValueError),
                     (x[:0], api.QuikError), (x[:1].expand(20, -1), api.QuikError), (x.cpu(), TypeError)):
        with pytest.raises(err):
            api.quik_linear_w4g(bad, w)
    with pytest.raises(TypeError):
        api.quik_linear_w4g(x, w, out=torch.empty((20, 96), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        api.quik_linear_w4g(x, w, out=torch.empty((20, 95), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        api.quik_linear_w4g(x, w, bias=torch.zeros(95, dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        api.quik_linear_w4g(x, w._replace(N=112))           # not what was packed
    w_q, scale = torch.zeros((16, 64), dtype=torch.uint8, device="cuda"), torch.ones((16, 1), dtype=torch.float16, device="cuda")
    for kw, err in ((dict(group=48), api.QuikError), (dict(group=64), ValueError), (dict(K=136, w_scale=scale.expand(16, 2).contiguous()), api.QuikError),
                    (dict(w_scale=scale.float()), TypeError), (dict(w_zero=scale), TypeError), (dict(w_scale=None), TypeError)):
        with pytest.raises(err):
            api.quik_weight_pack_w4g(**{**dict(w_q=w_q, w_scale=scale, K=128, group=128), **kw})
