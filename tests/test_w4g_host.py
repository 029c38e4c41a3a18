"""Layers with 4-bit weights in groups and layers of experts, host side: sizes, and bad arguments that come back as errors
before any launch.  No kernel is launched here, so no GPU is needed."""
import ctypes as C

import pytest

OK, EINVAL, ENULL, EALIGN, EUNSUPPORTED, EWORKSPACE = 0, -1, -2, -3, -4, -5
P, P256, ODD, NULL = C.c_void_p(0x1010), C.c_void_p(0x1000), C.c_void_p(0x1001), None     # never dereferenced


@pytest.fixture(scope="module")
def lib():
    from paper_2310_09259_amd import api
    return api.load()


def test_sizes(lib):
    # 16 x 128 tiles of 1 KB; a fp16 scale and an int8 zero point per channel and stored group, regions padded to 16 bytes
    assert lib.quik_w4g_bytes(16, 128, 128, 0, 0, 1) == 1024 + 32
    assert lib.quik_w4g_bytes(16, 128, 128, 1, 0, 1) == 1024 + 32 + 16
    assert lib.quik_w4g_bytes(17, 136, 32, 1, 0, 1) == 4 * (1024 + 16 * 4 * 3)
    assert lib.quik_w4g_bytes(17, 136, 256, 0, 0, 3) == lib.quik_w4g_bytes(17, 136, 0, 0, 0, 3) == 3 * 4 * (1024 + 32)
    assert lib.quik_w4g_bytes(34, 128, 64, 0, 1, 1) == 4 * (1024 + 64)                    # halves of 17 channels
    for bad in ((0, 128, 128, 0, 0, 1), (16, 0, 128, 0, 0, 1), (16, 12, 128, 0, 0, 1), (16, 128, 96, 0, 0, 1),
                (16, 128, 16, 0, 0, 1), (16, 128, -32, 0, 0, 1), (17, 128, 32, 0, 1, 1), (16, 128, 32, 2, 0, 1),
                (16, 128, 32, 0, 2, 1), (16, 128, 32, 0, 0, 0), (16, 128, 32, 0, 0, 1025), (16, 32776, 32, 0, 0, 1),
                ((1 << 20) + 1, 128, 32, 0, 0, 1)):
        assert lib.quik_w4g_bytes(*bad) == 0, bad
    few, many = lib.quik_moe_workspace_bytes(3, 4, 64, 0, 8, 0), lib.quik_moe_workspace_bytes(3, 4, 64, 0, 8, 1)
    assert few >= 4 * (8 + 2 + 12) and many >= few + 12 * 64 * 4
    assert lib.quik_moe_workspace_bytes(3, 4, 64, 1, 8, 1) < many
    for bad in ((0, 4, 64, 0, 8, 0), (3, 0, 64, 0, 8, 0), (3, 33, 64, 0, 8, 0), (3, 4, 0, 0, 8, 0), (3, 4, 63, 1, 8, 0),
                (3, 4, 64, 0, 0, 0), (3, 4, 64, 0, 1025, 0), (1 << 23, 4, 64, 0, 8, 0)):
        assert lib.quik_moe_workspace_bytes(*bad) == 0, bad


def _with(base, **changes):
    names = list(base)
    args = dict(base)
    for k, v in changes.items():
        assert k in names
        args[k] = v
    return [args[n] for n in names]


def test_pack_refuses_bad_arguments(lib):
    base = dict(w_q=P, ldw=64, w_scale=P, w_zero=NULL, N=16, K=128, group=32, glu=0, experts=1, w4=P, stream=NULL)
    for changes, rc in ((dict(N=0), EINVAL), (dict(K=-8), EINVAL), (dict(group=-1), EINVAL), (dict(glu=2), EINVAL),
                        (dict(glu=1, N=15), EINVAL), (dict(experts=0), EINVAL), (dict(ldw=48), EINVAL),
                        (dict(w_q=NULL), ENULL), (dict(w_scale=NULL), ENULL), (dict(w4=NULL), ENULL),
                        (dict(group=48), EUNSUPPORTED), (dict(group=96), EUNSUPPORTED), (dict(K=124), EUNSUPPORTED),
                        (dict(K=32776, ldw=32768), EUNSUPPORTED), (dict(experts=2000), EUNSUPPORTED),
                        (dict(ldw=72), EALIGN), (dict(w_q=ODD), EALIGN), (dict(w_scale=ODD), EALIGN), (dict(w4=ODD), EALIGN)):
        assert lib.quik_weight_pack_w4g(*_with(base, **changes)) == rc, changes


LINEAR = dict(type=0, x=P, T=4, K=128, ldx=128, w4=P, group=32, has_zero=0, glu=0, bias=NULL, N=16, y=P, ldy=16, stream=NULL)
PRODUCT_ERRORS = [
    (dict(type=2), EINVAL), (dict(type=-1), EINVAL), (dict(T=0), EINVAL), (dict(T=-1), EINVAL), (dict(K=0), EINVAL),
    (dict(ldx=120), EINVAL), (dict(ldy=15), EINVAL), (dict(N=0), EINVAL), (dict(has_zero=3), EINVAL), (dict(glu=-1), EINVAL),
    (dict(glu=1, N=17), EINVAL), (dict(x=NULL), ENULL), (dict(w4=NULL), ENULL), (dict(y=NULL), ENULL),
    (dict(group=33), EUNSUPPORTED), (dict(K=12, ldx=16), EUNSUPPORTED), (dict(K=40000, ldx=40000), EUNSUPPORTED),
    (dict(N=1 << 21, ldy=1 << 21), EUNSUPPORTED), (dict(x=ODD), EALIGN), (dict(ldx=132), EALIGN), (dict(w4=ODD), EALIGN),
    (dict(y=ODD), EALIGN), (dict(bias=ODD), EALIGN)]


@pytest.mark.parametrize("changes,rc", PRODUCT_ERRORS + [(dict(T=(1 << 24) + 1), EUNSUPPORTED), (dict(ldx=(1 << 22) + 8), EUNSUPPORTED)])
def test_linear_refuses_bad_arguments(lib, changes, rc):
    assert lib.quik_linear_w4g(*_with(LINEAR, **changes)) == rc


@pytest.mark.parametrize("changes,rc", PRODUCT_ERRORS + [
    (dict(top_k=0), EINVAL), (dict(top_k=33), EUNSUPPORTED), (dict(T=1 << 22, top_k=8), EUNSUPPORTED), (dict(experts=0), EINVAL),
    (dict(experts=1025), EUNSUPPORTED), (dict(x_per_slot=2), EINVAL), (dict(ids=NULL), ENULL), (dict(workspace=NULL), ENULL),
    (dict(ids=ODD), EALIGN), (dict(weights=ODD), EALIGN), (dict(workspace=P), EALIGN), (dict(workspace_bytes=16), EWORKSPACE),
    (dict(weights=P, workspace_bytes=256), EWORKSPACE),
    (dict(N=1 << 16, ldy=1 << 16, K=4096, ldx=4096, experts=1024), EUNSUPPORTED),      # 17 GB of scales
    (dict(T=1 << 20, top_k=2, ldx=2048), EUNSUPPORTED), (dict(T=1 << 19, top_k=2, ldx=2048, x_per_slot=1), EUNSUPPORTED)])
def test_experts_refuse_bad_arguments(lib, changes, rc):
    base = dict(type=0, x=P, ldx=128, x_per_slot=0, ids=P, weights=NULL, T=4, top_k=2, K=128, w4=P, group=32, has_zero=0,
                glu=0, bias=NULL, N=16, experts=8, y=P, ldy=16, workspace=P256, workspace_bytes=1 << 20, stream=NULL)
    assert lib.quik_moe_linear_w4g(*_with(base, **changes)) == rc


def test_router_refuses_bad_arguments(lib):
    base = dict(type=2, logits=P, T=4, experts=16, ldl=16, bias=NULL, score=0, groups=1, topk_groups=1, group_top=1, top_k=4,
                renormalize=1, scale=1.0, ids=P, weights=P, stream=NULL)
    for changes, rc in ((dict(type=3), EINVAL), (dict(score=2), EINVAL), (dict(renormalize=2), EINVAL), (dict(T=0), EINVAL),
                        (dict(experts=0), EINVAL), (dict(ldl=15), EINVAL), (dict(top_k=0), EINVAL), (dict(top_k=17), EINVAL),
                        (dict(groups=0), EINVAL), (dict(groups=3), EINVAL), (dict(topk_groups=0), EINVAL),
                        (dict(topk_groups=2), EINVAL), (dict(group_top=0), EINVAL), (dict(groups=4, group_top=5), EINVAL),
                        (dict(groups=8, topk_groups=1, top_k=3), EINVAL), (dict(logits=NULL), ENULL), (dict(ids=NULL), ENULL),
                        (dict(weights=NULL), ENULL), (dict(experts=1040, ldl=1040), EUNSUPPORTED),
                        (dict(experts=64, ldl=64, top_k=33), EUNSUPPORTED),
                        (dict(experts=130, ldl=130, groups=65, topk_groups=65), EUNSUPPORTED), (dict(logits=ODD), EALIGN),
                        (dict(bias=ODD), EALIGN), (dict(ids=ODD), EALIGN), (dict(weights=ODD), EALIGN)):
        assert lib.quik_moe_route(*_with(base, **changes)) == rc, changes


def test_binding_refuses_what_it_cannot_pass_on():
    """Host tensors and foreign objects, before the library is called."""
    import torch
    from paper_2310_09259_amd import api
    x = torch.zeros((2, 128), dtype=torch.float16)
    w = api.WeightW4G(torch.zeros(1056, dtype=torch.uint8), 16, 128, 128, False, False, 0)
    with pytest.raises(TypeError):
        api.quik_weight_pack_w4g(torch.zeros((16, 64), dtype=torch.uint8), torch.ones((16, 1), dtype=torch.float16), 128, 128)
    with pytest.raises(TypeError):
        api.quik_linear_w4g(x, w)
    with pytest.raises(TypeError):
        api.quik_linear_w4g(x, w.data)
    with pytest.raises(ValueError):
        api.quik_moe_linear_w4g(x, torch.zeros((2, 1), dtype=torch.int32), w)
    with pytest.raises(TypeError):
        api.quik_moe_route(torch.zeros((2, 8)), 2)
    with pytest.raises(ValueError):
        api.quik_moe_route(torch.zeros((2, 8)), 2, score="relu")


def test_kernel_choice(lib):
    """Which kernel a product runs on, at the borders of the rules, and what is refused."""
    form = lib.quik_debug_w4g_form
    cus = 256
    assert form(1, 4096, 4096, 0, 0, cus) == 0 and form(1, 4112, 4096, 0, 0, cus) == 1     # a block per CU, and one more
    assert form(1, 4096, 4096, 1, 0, cus) == 1                                             # halves go in pairs
    assert form(16, 8192, 4096, 0, 0, cus) == 1 and form(16, 8208, 4096, 0, 0, cus) == 2
    assert form(16, 24560, 4096, 0, 0, cus) == 2 and form(16, 24576, 4096, 0, 0, cus) == 3
    assert form(17, 4096, 4096, 0, 0, cus) == 4 and form(32, 11008, 4096, 0, 0, cus) == 5
    assert form(48, 11008, 4096, 0, 0, cus) == 6 and form(128, 11008, 4096, 0, 0, cus) == 7
    assert form(256, 11008, 4096, 0, 0, cus) == 8 and form(2048, 11008, 4096, 0, 0, cus) == 9
    assert form(4096, 28672, 8192, 0, 0, cus) == 10 and form(4096, 28672, 8192, 1, 0, cus) != 10
    assert form(64, 2816, 2048, 1, 64, cus) == 3 and form(65, 2816, 2048, 1, 64, cus) == 11    # a row at a time: up to one each
    assert form(6400, 2816, 2048, 1, 64, cus) == 11 and form(6401, 2816, 2048, 1, 64, cus) == 12
    for rows in list(range(1, 70)) + [127, 129, 300, 1000, 5000, 1 << 20]:
        for glu in (0, 1):
            for experts in (0, 8, 1024):
                assert 0 <= form(rows, 642, 904, glu, experts, cus) <= 12
    for bad, rc in (((0, 64, 64, 0, 0, cus), EINVAL), ((1, 0, 64, 0, 0, cus), EINVAL), ((1, 64, 12, 0, 0, cus), EUNSUPPORTED),
                    ((1, 63, 64, 1, 0, cus), EINVAL), ((1, 64, 64, 0, -1, cus), EINVAL), ((1, 64, 64, 0, 0, 0), EINVAL)):
        assert form(*bad) == rc, bad
    assert lib.quik_debug_set_w4g_form(13) == EINVAL and lib.quik_debug_set_w4g_form(-2) == EINVAL
    assert lib.quik_debug_set_w4g_form(3) == OK and lib.quik_debug_set_w4g_form(-1) == OK
