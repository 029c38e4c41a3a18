"""w4g layers at the ends of what is accepted: groups far longer than a row, and the widest and deepest layer."""
import numpy as np
import pytest

from tests.test_gpu_w4g import STEP, TINY, layer, pack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [4096, 1 << 20, 2 ** 31 - 128])
@pytest.mark.parametrize("K", [8, 136, 520])
@pytest.mark.parametrize("zero", [False, True])
def test_a_group_longer_than_the_row_is_one_for_the_row(group, K, zero):
    """The same bytes as group = 0; K + group - 1 is beyond 2^31 for the longest."""
    import torch
    raw = layer(K, 50, K, 0, zero)
    assert torch.equal(pack(raw, K, group).data, pack(raw, K, 0).data)
    experts = layer(K + 2, 18, K, 0, zero, experts=3)
    assert torch.equal(pack(experts, K, group).data, pack(experts, K, 0).data)


def test_the_widest_and_deepest_layer():
    """N = 2^20, K = 32768: 2^24 tiles to pack, 17 GB of weights, output rows of 2 MB.  Every channel has its own pattern of codes
    (a row shifted by its number); sampled channels are checked, the first and last of all among them.  Tolerance as in
    test_gpu_w4g, the sums' 2^-24 for each of K terms."""
    import torch
    from paper_2310_09259_amd import api
    N, K = 1 << 20, 32768
    ld = K // 2
    gen = torch.Generator(device="cuda").manual_seed(3)
    ring = torch.randint(0, 256, (ld + N // 64 + 64,), generator=gen, device="cuda", dtype=torch.uint8)
    w_q = torch.empty((N, ld), dtype=torch.uint8, device="cuda")
    for at in range(0, N, 1 << 16):                           # row n: the ring from n / 64 + n % 64 on
        n = torch.arange(at, at + (1 << 16), device="cuda")
        w_q[at:at + (1 << 16)] = torch.as_strided(ring, (N // 64, 64, ld), (1, 1, 1))[n // 64, n % 64]
    scale = (torch.rand((N, 1), generator=gen, device="cuda") * 0.015 + 0.005).half()
    w = api.quik_weight_pack_w4g(w_q, scale, K, 0)
    at = torch.tensor([0, 1, 15, 16, 4095, 4096, (1 << 19) - 1, 1 << 19, (1 << 19) + 17, N - 17, N - 16, N - 1], device="cuda")
    codes = w_q[at].cpu().numpy().astype(np.int64)
    q = np.stack((codes & 15, codes >> 4), -1).reshape(len(at), K)
    W = (q - 16 * (q > 7)) * scale[at].double().cpu().numpy()
    del w_q
    for T in (1, 20, 270):
        x = torch.randn((T, K), generator=gen, device="cuda").half()
        y = api.quik_linear_w4g(x, w)[:, at].double().cpu().numpy()
        xs = x.double().cpu().numpy()
        ref, tol = xs @ W.T, 2.0 ** -24 * (K + 8) * (np.abs(xs) @ np.abs(W).T)
        assert np.all(np.abs(y - ref) <= STEP["float16"] * (np.abs(ref) + tol) + tol + TINY["float16"]), T


def test_a_weighted_sum_of_2_to_the_34_outputs():
    """2^17 tokens of one slot and 2^17 channels: 2^32 groups of four columns to add up, 69 GB of sums in memory."""
    import torch
    from paper_2310_09259_amd import api
    T, K, N, E = 1 << 17, 128, 1 << 17, 2
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        torch.cuda.empty_cache()
    raw = layer(4, N, K, 128, False, experts=E)
    w = pack(raw, K, 128)
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((T, K), generator=gen, device="cuda").half()
    ids = torch.randint(0, E, (T, 1), generator=gen, device="cuda", dtype=torch.int32)
    weights = torch.rand((T, 1), generator=gen, device="cuda")
    y = api.quik_moe_linear_w4g(x, ids, w, weights=weights)
    for t in (0, 1, T // 2, T - 2, T - 1):
        ref = x[t].double().cpu().numpy() @ raw[3][ids[t, 0].item()].T * weights[t, 0].item()
        mag = np.abs(x[t].double().cpu().numpy()) @ np.abs(raw[3][ids[t, 0].item()]).T * weights[t, 0].item()
        tol = 2.0 ** -24 * (K + 16) * mag
        got = y[t].double().cpu().numpy()
        assert np.all(np.abs(got - ref) <= STEP["float16"] * (np.abs(ref) + tol) + tol + TINY["float16"]), t
    del y
    torch.cuda.empty_cache()
