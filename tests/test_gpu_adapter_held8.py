"""Gradients from activations in 8 bits whose tokens share blocks with others': what a value that is no number, or a large one, in a
padding token or another slot's token does to them, and what it does not."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import Problem, assert_within, held8

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Step:
    def __init__(self, dtype):
        # 400 tokens: the blocks' borders are 128, 256 and 384.  Slot 0 has tokens in the first two, slot 1 in the second, slot 2 in the rest
        self.p = p = Problem(dtype, 48, 72, 400, [8, 20, 5], 20, "none", seed=30)
        print("case", dtype, flush=True)
        p.slot_of[3:140:2], p.slot_of[140:256:3], p.slot_of[256:] = 0, 1, 2
        self.bank = pp.AdapterBank(p.m, p.k, 3, 20, pp.PP_F16 if dtype == "f16" else pp.PP_F32)
        self.bank.load_many(range(3), [dev(a) for a in p.a], [dev(b) for b in p.b], p.c)
        self.slot_of = dev(p.slot_of)
        self.u = self.bank.project(dev(p.x), self.slot_of)                    # the pass itself ran on sound values
        self.g = self.bank.grad_input(None, dev(p.dy), self.slot_of)

    def weights(self, x):
        return self.bank.grad_weights(pp.act8_pack(dev(x)), self.u, self.g.g, self.g.v, self.slot_of, torch.arange(3, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_block_that_is_not_finite_spoils_its_row_for_every_slot_in_it(dtype, bad):
    s = Step(dtype)
    p = s.p
    da0, db0 = s.weights(p.x)
    for token, spoilt in ((4, [0]), (128, [0, 1]), (140, [0, 1]), (255, [0, 1]), (384, [2])):   # padding, padding, slot 1's, padding, slot 2's
        x = p.x.copy()
        x[7, token] = bad
        da, db = s.weights(x)
        for slot in range(3):
            rest = [c for c in range(p.k) if c != 7 or slot not in spoilt]
            assert torch.equal(da[slot][:, rest], da0[slot][:, rest]), (token, slot)
            if slot in spoilt:
                assert torch.isnan(da[slot, : p.ranks[slot], 7]).all() and not da[slot, p.ranks[slot]:, 7].any(), (token, slot)
        assert torch.equal(db, db0)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_padding_that_was_set_to_zero_spoils_nothing(dtype):
    s = Step(dtype)
    p = s.p
    x = p.x.copy()
    x[:, p.slot_of < 0] = 0
    da, db = s.weights(x)
    (_, want_a, want_b), (_, room_a, room_b) = p.backward(held8(x), None, range(3))
    assert_within(da.cpu().numpy(), want_a, room_a, "dA")
    assert_within(db.cpu().numpy(), want_b, room_b, "dB")
    assert torch.isfinite(da).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_large_value_coarsens_its_block(dtype):
    """The step is that of the block's largest value, whoever's: gradients are those of the values held."""
    s = Step(dtype)
    p = s.p
    x = p.x.copy()
    x[7, 130] = 30000.0                                                       # a padding token's
    da, db = s.weights(x)
    (_, want_a, want_b), (_, room_a, room_b) = p.backward(held8(x), None, range(3))
    assert_within(da.cpu().numpy(), want_a, room_a, "dA")
    assert_within(db.cpu().numpy(), want_b, room_b, "dB")
