"""Layers of as many experts as a lane's worth of the plan holds, one more, and the limit: by the plan (rows > experts) and a row
or token at a time (rows <= experts), against the definition."""
import numpy as np
import pytest

from tests.test_gpu_moe import moe_reference
from tests.test_gpu_w4g import activations, check, layer, pack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,glu,combine", [("float16", False, True), ("bfloat16", True, False), ("bfloat16", False, True)])
@pytest.mark.parametrize("E,T,top_k", [(63, 40, 3), (64, 40, 3), (64, 32, 2), (65, 33, 2), (128, 50, 4), (129, 200, 2), (1024, 300, 4),
                                       (1024, 128, 8)])
def test_many_experts(dtype, glu, combine, E, T, top_k):
    """The first, the last and the experts on both sides of every 64th are chosen for certain; runs of them are not chosen."""
    import torch
    from paper_2310_09259_amd import api
    K, N = 136, 34
    raw = layer(E + T, N, K, 64, True, experts=E)
    w = pack(raw, K, 64, glu)
    rng = np.random.Generator(np.random.PCG64(E))
    ids = rng.integers(-1, E + 1, (T, top_k)).astype(np.int32)
    ids[(ids > 70) & (ids < 110)] = -1
    sure = [e for k in range(0, E + 64, 64) for e in (k - 1, k) if 0 <= e < E] + [E - 1]
    ids.reshape(-1)[rng.permutation(T * top_k)[:len(sure)]] = sure
    weights = rng.uniform(0.1, 1.0, (T, top_k)).astype(np.float32)
    x = activations(E, T, K, dtype)
    y = api.quik_moe_linear_w4g(x, torch.from_numpy(ids).cuda(), w, weights=torch.from_numpy(weights).cuda() if combine else None)
    ref, tol = moe_reference(x.double().cpu().numpy(), ids, raw[3], raw[4], dtype, top_k, glu, weights=weights if combine else None)
    check(y, ref, tol, dtype)
