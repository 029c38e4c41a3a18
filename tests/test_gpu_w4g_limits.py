"""w4g layers at the ends of what is accepted: groups far longer than a row."""
import pytest

from tests.test_gpu_w4g import layer, pack

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
