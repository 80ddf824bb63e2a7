"""Refusals of loading several slots in one call (no GPU): a host-only bank and addresses that nothing reads."""
import pytest

import paper_2206_10620_amd as pp


@pytest.fixture
def bank():
    st, h = pp.pp_adapter_plan(64, 32, 4, 8, pp.PP_F16, pp.PP_FLAG_HOST_ONLY)
    assert st == pp.PP_OK
    yield h
    pp.pp_adapter_destroy(h)


def load(bank, **kw):
    entries = {**dict(slots=[0, 3, 1], ranks=[8, 1, 0], scales=[1.0, -2.0, 0.0], a=[16, 32, 0], b=[48, 64, 0]), **kw}
    return pp.pp_adapter_load_many(bank, *entries.values())


def test_lists_that_are_in_order_get_as_far_as_the_device(bank):
    assert load(bank) == pp.PP_ERR_UNSUPPORTED                                             # the bank is host-only
    assert load(bank, slots=[2, 2, 2]) == pp.PP_ERR_UNSUPPORTED                            # a slot may be listed again


def test_every_entry_is_checked(bank):
    for bad in (dict(slots=[0, 4, 1]), dict(slots=[0, 3, -1]), dict(ranks=[9, 1, 0]), dict(ranks=[8, -1, 0])):
        assert load(bank, **bad) == pp.PP_ERR_SHAPE, bad
    for bad in (dict(a=[16, 0, 0]), dict(b=[0, 64, 0]), dict(ranks=[8, 1, 1])):
        assert load(bank, **bad) == pp.PP_ERR_NULL, bad
    for scale in (float("inf"), float("-inf"), float("nan"), 1e39):                        # the last one is none in binary32
        assert load(bank, scales=[1.0, scale, 0.0]) == pp.PP_ERR_UNSUPPORTED
    for bad in (dict(a=[16, 34, 0]), dict(b=[40, 64, 0])):
        assert load(bank, **bad) == pp.PP_ERR_ALIGN, bad


def test_arrays_and_counts(bank):
    assert load(None) == pp.PP_ERR_NULL
    f = pp.lib().pp_adapter_load_many                                                      # (tests that reach the arrays are above)
    assert load(bank, slots=[], ranks=[], scales=[], a=[], b=[]) in (pp.PP_ERR_NULL, pp.PP_ERR_SHAPE)
    for i in range(2, 7):
        args = [bank, 1, 64, 64, 64, 64, 64, None]
        args[i] = None
        assert f(*args) == pp.PP_ERR_NULL
    assert f(bank, 0, 64, 64, 64, 64, 64, None) == f(bank, -1, 64, 64, 64, 64, 64, None) == pp.PP_ERR_SHAPE
    with pytest.raises(AssertionError):
        load(bank, ranks=[8, 1])
