"""Products of more threads than a grid takes are refused before anything is launched (host only)."""
import ctypes as C

import pytest

P, P256 = C.c_void_p(0x1010), C.c_void_p(0x1000)     # never dereferenced
EUNSUPPORTED = -4


@pytest.mark.parametrize("glu,combine", [(0, False), (0, True), (1, True)])
def test_a_row_at_a_time_of_the_widest_experts(glu, combine):
    """1024 rows of 2^20 channels, 64 to a workgroup of 256 threads: 2^32."""
    from paper_2310_09259_amd import api
    lib = api.load()
    N, K, experts, T = 1 << 20, 128, 1024, 1024
    assert lib.quik_debug_moe_w4g_form(T, 1, N, K, 128, glu, experts, int(combine), 256) == 3
    need = lib.quik_moe_workspace_bytes(T, 1, N, glu, experts, int(combine))
    assert need > 0
    rc = lib.quik_moe_linear_w4g(0, P256, K, 0, P, P if combine else None, T, 1, K, P256, 128, 0, glu, None, N, experts, P, N, P256,
                                 need, None)
    assert rc == EUNSUPPORTED


def test_the_same_of_a_layer():
    """2^24 tokens of 2^20 channels, 512 threads to 256 x 256 outputs."""
    from paper_2310_09259_amd import api
    rc = api.load().quik_linear_w4g(0, P256, 1 << 24, 128, 128, P256, 128, 0, 0, None, 1 << 20, P, 1 << 20, None)
    assert rc == EUNSUPPORTED
