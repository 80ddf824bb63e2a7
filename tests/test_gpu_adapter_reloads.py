"""Slots that are loaded again between a forward pass, the first and the second half of the backward pass: the gradients are those of
what the passes ran with, and nothing is read of u and v that they did not write."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import Problem, assert_within, held8

pytestmark = pytest.mark.gpu
PP = {"f16": pp.PP_F16, "f32": pp.PP_F32}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def poisoned(nbytes):
    """Memory in which every binary32 value is a NaN."""
    return torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")


class Step:
    """The calls of a tuning step one by one, on buffers that hold NaN before."""

    def __init__(self, p, held=False):
        print("case", p.dtype, p.m, p.k, p.n, p.ranks, p.max_rank, held, flush=True)
        self.p = p
        self.bank = pp.AdapterBank(p.m, p.k, p.slots, p.max_rank, PP[p.dtype])
        for s, r in enumerate(p.ranks):
            if r:
                self.load(s, p.a[s], p.b[s], p.c[s])
        self.x, self.dy, self.slot_of = dev(p.x), dev(p.dy), dev(p.slot_of)
        self.held = pp.act8_pack(self.x).buffer if held else None
        h, n = self.bank.handle, p.n
        self.u, self.v = poisoned(pp.pp_adapter_u_bytes(h, n)), poisoned(pp.pp_adapter_v_bytes(h, n))
        self.stream = torch.cuda.current_stream().cuda_stream

    def load(self, s, a, b, c):
        self.bank.load(s, dev(a), dev(b), c)

    def project(self):
        assert pp.pp_adapter_project(self.bank.handle, self.x.data_ptr(), self.slot_of.data_ptr(), self.u.data_ptr(), self.p.n, self.stream) == pp.PP_OK

    def grad_input(self):
        assert pp.pp_adapter_grad_input(self.bank.handle, None, self.dy.data_ptr(), None, None, self.slot_of.data_ptr(), self.v.data_ptr(), None, self.p.n,
                                        self.stream) == pp.PP_OK

    def grad_weights(self):
        p, h = self.p, self.bank.handle
        which = torch.arange(p.slots, dtype=torch.int32, device="cuda")
        da = poisoned(p.slots * p.max_rank * p.k * 4).view(torch.float32).view(p.slots, p.max_rank, p.k)
        db = poisoned(p.slots * p.max_rank * p.m * 4).view(torch.float32).view(p.slots, p.m, p.max_rank)
        work = poisoned(pp.pp_adapter_work_bytes(h, p.n, p.slots))
        x = self.x if self.held is None else self.held
        assert pp.pp_adapter_grad_weights(h, x.data_ptr(), int(self.held is not None), self.u.data_ptr(), self.dy.data_ptr(), self.v.data_ptr(),
                                          self.slot_of.data_ptr(), which.data_ptr(), p.slots, da.data_ptr(), db.data_ptr(), work.data_ptr(), p.n,
                                          self.stream) == pp.PP_OK
        return da, db


def another(p, rank, seed):
    """An adapter of another rank for any slot."""
    rs = np.random.RandomState(seed)
    dt = p.x.dtype
    return rs.standard_normal((rank, p.k)).astype(dt), rs.standard_normal((p.m, rank)).astype(dt), 1.75


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m,k,n", [(48, 65, 77), (200, 130, 700), (256, 192, 4096)], ids=str)
def test_loading_between_the_halves_changes_nothing(m, k, n, dtype, held):
    """A larger rank, a smaller one, an emptied slot, another factor alone, and a slot that was empty when the passes ran."""
    p = Problem(dtype, m, k, n, [8, 24, 5, 16, 0], 40, "mixed", seed=n)
    s = Step(p, held)
    s.project()
    s.grad_input()
    want = s.grad_weights()
    (_, da, db), (_, da_bound, db_bound) = p.backward(held8(p.x) if held else p.x, None, range(p.slots))
    assert_within(want[0].cpu().numpy(), da, da_bound, "dA")
    assert_within(want[1].cpu().numpy(), db, db_bound, "dB")
    s.load(0, *another(p, 40, 1))
    s.load(1, *another(p, 3, 2))
    s.bank.unload(2)
    s.load(3, p.a[3], p.b[3], -p.c[3])
    s.load(4, *another(p, 40, 3))
    got = s.grad_weights()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_loading_before_the_backward_pass(dtype):
    """u as it was, v of what is there now: dB of the one, dA of the other."""
    p = Problem(dtype, 96, 80, 300, [8, 24, 0], 40, "runs", seed=2)
    s = Step(p)
    s.project()
    before = p.backward(p.x, None, range(3))
    for slot, rank in ((0, 33), (1, 4), (2, 16)):
        p.a[slot], p.b[slot], p.c[slot] = another(p, rank, slot)
        p.ranks[slot] = rank
        s.load(slot, p.a[slot], p.b[slot], p.c[slot])
    s.grad_input()
    after = p.backward(p.x, None, range(3))
    da, db = s.grad_weights()
    assert_within(da.cpu().numpy(), after[0][1], after[1][1], "dA")
    assert_within(db.cpu().numpy(), before[0][2], before[1][2], "dB")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_tokens_named_for_another_slot_since_count_for_neither(dtype):
    """u and v of such a token are the old slot's: it is left out of both sums, and of no other's."""
    p = Problem(dtype, 64, 50, 300, [8, 24, 5], 24, "mixed", seed=6)
    s = Step(p)
    s.project()
    s.grad_input()
    old = p.slot_of.copy()
    p.slot_of[:200:3] = (p.slot_of[:200:3] + 2) % 4 - 1                        # the next one, or none after the last
    s.slot_of.copy_(dev(p.slot_of))
    da, db = s.grad_weights()
    p.slot_of[p.slot_of != old] = -1
    (_, want_a, want_b), (_, room_a, room_b) = p.backward(p.x, None, range(3))
    assert_within(da.cpu().numpy(), want_a, room_a, "dA")
    assert_within(db.cpu().numpy(), want_b, room_b, "dB")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_slot_far_behind_the_first_tokens(dtype):
    """Blocks are found 64 at a time: a slot whose first token is in the second of those runs, and one that has tokens in each of three."""
    p = Problem(dtype, 33, 40, 20000, [6, 17, 9], 20, "none", seed=4)
    p.slot_of[8192 + 130: 8192 + 140] = 0
    p.slot_of[[5, 9000, 19999]] = 1
    s = Step(p)
    s.project()
    s.grad_input()
    da, db = s.grad_weights()
    (_, want_a, want_b), (_, room_a, room_b) = p.backward(p.x, None, range(3))
    assert_within(da.cpu().numpy(), want_a, room_a, "dA")
    assert_within(db.cpu().numpy(), want_b, room_b, "dB")
    assert not da[2].any() and not db[2].any()
