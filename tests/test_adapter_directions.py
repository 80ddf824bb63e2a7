"""A square layer's plan and the plan of its transposed weights have the same sizes: each is taken in its own direction only."""
import numpy as np
import pytest

import synth
import paper_2206_10620_amd as pp

H = pp.PP_FLAG_HOST_ONLY
AT = [i << 20 for i in range(1, 8)]              # addresses that a host-only bank does not touch


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_plan_of_the_other_direction_is_refused(dtype):
    code = pp.PP_F16 if dtype == "f16" else pp.PP_F32
    st, bank = pp.pp_adapter_plan(48, 48, 2, 8, code, H)
    assert st == pp.PP_OK
    lay = synth.random_block_layer("square", 48, 48, 8, 16, 16, dtype, 0.5, 0.5, 3, relu=True)
    plan, plan_t = pp.block_plan_from_layer(lay, host_only=True), pp.block_plan_transposed_from_layer(lay, host_only=True)
    run = lambda p: pp.pp_adapter_run(bank, p.handle, AT[0], AT[1], AT[2], AT[3], 8)
    grad = lambda p, dx=AT[3]: pp.pp_adapter_grad_input(bank, p.handle, AT[0], None, None, AT[1], AT[2], dx, 8)
    assert run(plan_t) == grad(plan) == pp.PP_ERR_SHAPE
    assert run(plan) == grad(plan_t) == pp.PP_ERR_UNSUPPORTED        # in order, but host-only
    assert grad(plan, None) == pp.PP_ERR_UNSUPPORTED                 # no dx: no plan is looked at
    plan.close()
    plan_t.close()
    pp.pp_adapter_destroy(bank)


def test_what_a_refused_plan_would_have_given_is_another_matrix():
    """The two directions differ, on a square layer too: the transposed plan holds the transpose and no bias or ReLU."""
    lay = synth.random_block_layer("square", 48, 48, 8, 16, 16, "f16", 0.5, 0.5, 3, relu=True)
    plan, plan_t = pp.block_plan_from_layer(lay, host_only=True), pp.block_plan_transposed_from_layer(lay, host_only=True)
    (_, w), (_, wt) = pp.pp_block_gemm_unpack(plan.handle, 0, 64, 48), pp.pp_block_gemm_unpack(plan_t.handle, 0, 64, 48)
    assert np.array_equal(w[:48], wt[:48].T) and not np.array_equal(w, wt)
    plan.close()
    plan_t.close()
