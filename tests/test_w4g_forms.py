"""Which kernel a w4g product of experts runs on (host only): what the hook says is what the launch resolves to, for weighted
products by the token too, and with a form that was set."""
import pytest

OK, EINVAL, EUNSUPPORTED = 0, -1, -4
CUS = 256


@pytest.fixture
def lib():
    from paper_2310_09259_amd import api
    yield api.load()
    api.load().quik_debug_set_w4g_form(-1)


def test_weighted_products_go_by_their_tokens(lib):
    """A token and its slots are one workgroup's work: the choice goes by the tokens' channel blocks, not the slots'."""
    form = lib.quik_debug_moe_w4g_form
    # 4 tokens, 8 slots, 64 experts: 4 x 128 channel blocks, two to a CU; without weights 32 x 128
    assert form(4, 8, 2048, 1408, 128, 0, 64, 1, CUS) == 1 and form(4, 8, 2048, 1408, 128, 0, 64, 0, CUS) == 3
    assert form(4, 8, 2048, 1408, 128, 1, 64, 1, CUS) == 3              # paired halves go row by row, and are added up
    assert form(2, 8, 2048, 1408, 128, 0, 64, 1, CUS) == 0              # a block to a CU
    assert form(8, 8, 2048, 1408, 128, 0, 64, 1, CUS) == 2              # up to as many rows as experts
    assert form(9, 8, 2048, 1408, 128, 0, 64, 1, CUS) == 11             # more: by the plan
    for T in (1, 3, 8, 9, 500, 900):
        for glu in (0, 1):
            assert form(T, 8, 2048, 1408, 64, glu, 64, 0, CUS) == lib.quik_debug_w4g_form(T * 8, 2048, 1408, glu, 64, CUS)


def test_a_form_that_was_set_shows_where_it_can_run(lib):
    moe, dense = lib.quik_debug_moe_w4g_form, lib.quik_debug_w4g_form
    for f in range(13):
        assert lib.quik_debug_set_w4g_form(f) == OK
        assert dense(300, 512, 512, 0, 0, CUS) == f
        assert dense(300, 512, 512, 1, 0, CUS) == {0: 1, 10: 9}.get(f, f)                  # no single blocks, no 256 x 256
        by_plan = moe(300, 2, 512, 512, 32, 0, 8, 1, CUS)
        assert by_plan == (11 if f < 6 else 9 if f == 10 else f)
        by_row = moe(2, 2, 512, 512, 32, 0, 8, 1, CUS)
        assert by_row == (f if f <= 3 else 2)


def test_refusals(lib):
    good = [4, 8, 2048, 1408, 128, 0, 64, 1, CUS]
    for at, value, rc in ((0, 0, EINVAL), (1, 0, EINVAL), (1, 33, EUNSUPPORTED), (2, 0, EINVAL), (3, 12, EUNSUPPORTED),
                          (4, 48, EUNSUPPORTED), (5, 2, EINVAL), (6, 0, EINVAL), (6, 1025, EUNSUPPORTED), (7, 2, EINVAL),
                          (8, 0, EINVAL)):
        assert lib.quik_debug_moe_w4g_form(*[value if i == at else v for i, v in enumerate(good)]) == rc, (at, value)
