"""Every kernel of the w4g products applies the scales in fp32 to exact products: nothing is rounded to 16 bits but the
output.  Rows of x with a single value make that visible: y = x_k s (q - z) is one product, whose 11 + 8 bits fp32 holds, times
a scale, and rounded once to the output's type (u = half a step).  In between at most eight roundings of 2^-24: one where sums
of a group are multiplied by their scale; where sums are in units of a scale, two for each of the three further groups of a row
of 392 columns (the quotient, the product), the units at the end being one more.  bf16 in kernels whose waves split K runs on
x (q + 136) - x (136 + z), both of at most 17 bits and so exact as well."""
import numpy as np
import pytest

from tests.test_gpu_w4g import STEP, TINY, activations, forced, layer, pack  # noqa: F401

pytestmark = pytest.mark.gpu


def _single(T, K, dtype, seed):
    """Rows of zeros with one value of all its bits -> x on the GPU, its columns."""
    import torch
    rng = np.random.Generator(np.random.PCG64(seed))
    at = rng.integers(0, K, T)
    x = torch.zeros((T, K), dtype=getattr(torch, dtype))
    x[torch.arange(T), torch.from_numpy(at)] = torch.from_numpy(rng.uniform(0.5, 2.0, T)).to(x.dtype)
    return x.cuda(), at


def _once_rounded(y, ref, dtype):
    y = y.double().cpu().numpy()
    limit = STEP[dtype] * np.abs(ref) * (1 + 2.0 ** -10) + TINY[dtype]
    err = np.abs(y - ref)
    assert np.all(err <= limit), float(np.nanmax(err / limit))


@pytest.mark.parametrize("form", range(13))
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("group,zero", [(32, True), (64, False), (64, True), (128, False), (128, True), (0, True)])
@pytest.mark.parametrize("T", [16, 300])
def test_weights_are_not_rounded(forced, form, dtype, group, zero, T):
    import torch
    from paper_2310_09259_amd import api
    K, N = 392, 274
    raw = layer(form, N, K, group, zero)
    w = pack(raw, K, group)
    x, at = _single(T, K, dtype, form + T)
    value = x[torch.arange(T), torch.from_numpy(at)].double().cpu().numpy()
    forced(form)
    y = api.quik_linear_w4g(x, w)
    _once_rounded(y, value[:, None] * raw[3].T[at], dtype)


@pytest.mark.parametrize("form", range(6, 13))
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("group", [32, 128])
def test_paired_halves_of_unrounded_weights(forced, form, dtype, group):
    """silu(gate) * value of exact factors: the exponential and the reciprocal are good to 2^-19 of it."""
    import torch
    from paper_2310_09259_amd import api
    T, K, N = 280, 264, 260
    raw = layer(form + 1, N, K, group, True)
    w = pack(raw, K, group, glu=True)
    x, at = _single(T, K, dtype, form)
    value = x[torch.arange(T), torch.from_numpy(at)].double().cpu().numpy()
    forced(form)
    y = api.quik_linear_w4g(x, w).double().cpu().numpy()
    a = value[:, None] * raw[3].T[at]
    g, v = a[:, :N // 2], a[:, N // 2:]
    ref = g / (1.0 + np.exp(-g)) * v
    assert np.all(np.abs(y - ref) <= (STEP[dtype] * (1 + 2.0 ** -10) + 2.0 ** -18) * np.abs(ref) + TINY[dtype])


@pytest.mark.parametrize("form", range(13))
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("group,scale", [(32, 6000.0), (64, 60000.0), (128, 65504.0), (128, 2.0 ** -24)])
def test_scales_at_the_ends_of_fp16(forced, form, dtype, group, scale):
    """s (q - z) beyond fp16's range, in a product that is not: as finite in one kernel as in another."""
    import torch
    from paper_2310_09259_amd import api
    T, K, N = 300, 264, 146
    w_q, s, z, _, wide = layer(2 * form, N, K, group, True)
    s = (np.random.Generator(np.random.PCG64(9)).uniform(0.5, 1.0, s.shape) * scale).astype(np.float16)
    of = np.arange(K) // group
    q = (w_q[..., :K // 2, None] >> np.array([0, 4])) & 15
    q = q.reshape(N, K).astype(np.int64)
    q = q - 16 * (q > 7) - z.astype(np.int64)[:, of]
    W = q * s.astype(np.float64)[:, of]
    w = pack((w_q, s, z), K, group)
    x, at = _single(T, K, dtype, form)
    x *= 2.0 ** -12 if scale > 1 else 1.0
    value = x[torch.arange(T), torch.from_numpy(at)].double().cpu().numpy()
    forced(form)
    _once_rounded(api.quik_linear_w4g(x, w), value[:, None] * W.T[at], dtype)


@pytest.mark.parametrize("form", range(13))
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("group", [32, 128, 256])
def test_scales_that_change_vanish_and_turn_within_a_channel(forced, form, dtype, group):
    """Scales over a range of 2^20, of both signs, a third of them 0, and a channel whose first or last ones are.  Tolerance: K
    terms and, for each of the G stored groups, four roundings of the sum so far, each 2^-24 of the absolute products."""
    import torch
    from paper_2310_09259_amd import api
    T, K, N = 290, 1160, 274
    rng = np.random.Generator(np.random.PCG64(form + group))
    w_q, s, z, _, _ = layer(form, N, K, group, True)
    s = (2.0 ** rng.uniform(-14, 6, s.shape) * rng.choice([-1.0, 1.0], s.shape)).astype(np.float16)
    s[rng.random(s.shape) < 0.33] = 0
    s[3, 0] = s[4, -1] = s[5, :2] = s[6, -2:] = 0
    s[7] = 0
    q = ((w_q[..., :K // 2, None] >> np.array([0, 4])) & 15).reshape(N, K).astype(np.int64)
    of = np.arange(K) // group
    q = q - 16 * (q > 7) - z.astype(np.int64)[:, of]
    W = q * s.astype(np.float64)[:, of]
    wide = np.abs(s.astype(np.float64))[:, of] * (np.abs(q) + 136.0) if dtype == "bfloat16" else np.abs(W)
    w = pack((w_q, s, z), K, group)
    x = activations(form, T, K, dtype)
    forced(form)
    y = api.quik_linear_w4g(x, w).double().cpu().numpy()
    xs = x.double().cpu().numpy()
    ref = xs @ W.T
    tol = 2.0 ** -24 * (K + 8 + 4 * 40) * (np.abs(xs) @ wide.T)
    assert np.all(np.abs(y - ref) <= STEP[dtype] * (np.abs(ref) + tol) + tol + TINY[dtype])
    assert np.all(y[:, 7] == 0)


@pytest.mark.parametrize("form", [2, 8, 9, 10])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_scale_that_is_no_number_spoils_its_own_channel_only(forced, form, bad):
    import torch
    from paper_2310_09259_amd import api
    T, K, N = 270, 392, 272
    w_q, s, z, W, _ = layer(8, N, K, 128, True)
    x, at = _single(T, K, "float16", 5)
    value = x[torch.arange(T), torch.from_numpy(at)].double().cpu().numpy()
    s[17, 1] = s[200, 3] = bad
    w = pack((w_q, s, z), K, 128)
    forced(form)
    keep = [n for n in range(N) if n not in (17, 200)]
    _once_rounded(api.quik_linear_w4g(x, w)[:, keep], value[:, None] * W.T[at][:, keep], "float16")


@pytest.mark.parametrize("form", range(13))
@pytest.mark.parametrize("d", [1.0, 2.0 ** 12])
def test_the_largest_bf16_activations(forced, form, d):
    """Up to 2^104 / d, d the largest quotient of two scales of a channel: no sum leaves fp32.  Tolerance as above."""
    import torch
    from paper_2310_09259_amd import api
    T, K, N = 260, 4096, 40
    rng = np.random.Generator(np.random.PCG64(form))
    w_q, s, z, _, _ = layer(form, N, K, 128, True)
    s = np.where(rng.random(s.shape) < 0.5, 1.0, d).astype(np.float16) * np.float16(2.0 ** -12)
    q = ((w_q[..., :K // 2, None] >> np.array([0, 4])) & 15).reshape(N, K).astype(np.int64)
    of = np.arange(K) // 128
    q = q - 16 * (q > 7) - z.astype(np.int64)[:, of]
    W = q * s.astype(np.float64)[:, of]
    w = pack((w_q, s, z), K, 128)
    x = activations(form, T, K, "bfloat16").clamp(-1, 1) * (2.0 ** 103 / d)
    forced(form)
    y = api.quik_linear_w4g(x, w).double().cpu().numpy()
    xs = x.double().cpu().numpy()
    ref = xs @ W.T
    tol = 2.0 ** -24 * (K + 8 + 4 * 32) * (np.abs(xs) @ (np.abs(s.astype(np.float64))[:, of] * (np.abs(q) + 136.0)).T)
    assert np.isfinite(y).all() and np.all(np.abs(y - ref) <= STEP["bfloat16"] * (np.abs(ref) + tol) + tol)


@pytest.mark.parametrize("form", range(13))
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_rows_that_are_no_numbers_spoil_no_other_row(forced, form, dtype):
    import torch
    from paper_2310_09259_amd import api
    T, K, N = 300, 392, 272
    w = pack(layer(form, N, K, 128, True), K, 128)
    x = activations(3, T, K, dtype)
    forced(form)
    clean = api.quik_linear_w4g(x, w)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    for t, v in ((0, float("nan")), (17, float("inf")), (140, -float("inf")), (299, float("nan"))):
        x[t, t % 128::5] = v
        keep[t] = False
    assert torch.equal(api.quik_linear_w4g(x, w)[keep], clean[keep])
