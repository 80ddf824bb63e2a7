"""Gradients of more slots than the scratch memory holds at once."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import Problem, assert_within, held8

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("dtype,held", [("f16", True), ("f32", False)])
def test_gradients_of_long_lists_in_parts(dtype, held):
    """4096 tokens and ranks up to 128 take 4 MB a slot: 61 slots at a time.  Of 140 listed ones each is right, in whichever part it is."""
    ranks = [1 + (7 * i) % 128 for i in range(70)]
    p = Problem(dtype, 40, 56, 4096, ranks, 128, "mixed", seed=40)
    print("case", dtype, held, flush=True)
    code = pp.PP_F16 if dtype == "f16" else pp.PP_F32
    bank = pp.AdapterBank(p.m, p.k, p.slots, 128, code)
    bank.load_many(range(70), [dev(a) for a in p.a], [dev(b) for b in p.b], p.c)
    which = [(3 * i) % 70 for i in range(70)] + [i if i % 5 else -1 for i in range(70)]
    assert pp.pp_adapter_work_bytes(bank.handle, p.n, len(which)) <= 1 << 28
    x, slot_of = dev(p.x), dev(p.slot_of)
    u = bank.project(x, slot_of)
    g = bank.grad_input(None, dev(p.dy), slot_of)
    da, db = bank.grad_weights(pp.act8_pack(x) if held else x, u, g.g, g.v, slot_of, dev(np.array(which, np.int32)))
    (_, want_a, want_b), (_, room_a, room_b) = p.backward(held8(p.x) if held else p.x, None, which)
    assert_within(da.cpu().numpy(), want_a, room_a, "dA")
    assert_within(db.cpu().numpy(), want_b, room_b, "dB")
    again = bank.grad_weights(pp.act8_pack(x) if held else x, u, g.g, g.v, slot_of, dev(np.array(which, np.int32)))
    assert torch.equal(da, again[0]) and torch.equal(db, again[1])
