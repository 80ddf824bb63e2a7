"""Loading several slots of an adapter bank in one call against loading them one by one: the products that follow have equal bits."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import Problem, assert_within

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def case(dtype, m, k, n, ranks, max_rank, seed):
    print("case", dtype, m, k, n, len(ranks), max_rank, flush=True)
    p = Problem(dtype, m, k, n, ranks, max_rank, "mixed", seed=seed)
    return p, pp.block_plan_from_layer(p.layer), pp.block_plan_transposed_from_layer(p.layer), [dev(t) for t in p.a], [dev(t) for t in p.b]


def outputs(p, bank, plan, plan_t):
    """Everything that reads a bank: both projections, both expansions, the factors."""
    x, slot_of = dev(p.x), dev(p.slot_of)
    y, u = bank.run(plan, x, slot_of, keep=True)
    g = bank.grad_input(plan_t, dev(p.dy), slot_of)
    return (y, g.dx) + tuple(bank.grad_weights(x, u, g.g, g.v, slot_of, torch.arange(p.slots, dtype=torch.int32, device="cuda")))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("ranks,max_rank", [([3], 8), ([16, 0, 33, 64, 1], 64), ([1 + i % 20 for i in range(64)], 20), ([i % 19 for i in range(131)], 18)],
                         ids=["one", "few", "a launch", "three launches"])
def test_it_is_one_load_after_another(ranks, max_rank, dtype):
    p, plan, plan_t, a, b = case(dtype, 130, 100, 150, ranks, max_rank, 1)
    banks = [pp.AdapterBank(p.m, p.k, p.slots, max_rank, plan.dtype) for _ in range(2)]
    some = [s for s in range(p.slots) if ranks[s]]
    for s in some:
        banks[0].load(s, a[s], b[s], p.c[s])
    order = some[::-1]                                                          # in any order of slots
    banks[1].load_many(order, [a[s] for s in order], [b[s] for s in order], [p.c[s] for s in order])
    want, got = outputs(p, banks[0], plan, plan_t), outputs(p, banks[1], plan, plan_t)
    for t, w in zip(got, want):
        assert torch.equal(t, w)
    y, bound = p.forward()
    assert_within(got[0].cpu().numpy(), y, bound, "y")


def test_a_slot_listed_again_holds_its_last_entry_and_rank_0_empties_it():
    p, plan, plan_t, a, b = case("f16", 64, 80, 60, [16, 5, 9], 16, 2)
    bank, other = pp.AdapterBank(64, 80, 3, 16), pp.AdapterBank(64, 80, 3, 16)
    none = (a[0][:0], b[0][:, :0].contiguous())
    bank.load_many([0, 1, 0, 2, 1, 2], [a[1], a[0], a[0], a[2], a[1], none[0]], [b[1], b[0], b[0], b[2], b[1], none[1]], [9.0, 9.0, p.c[0], 9.0, p.c[1], 1.0])
    for s in (0, 1):
        other.load(s, a[s], b[s], p.c[s])
    for t, w in zip(outputs(p, bank, plan, plan_t), outputs(p, other, plan, plan_t)):
        assert torch.equal(t, w)


def test_a_list_with_a_refused_entry_loads_nothing():
    p, plan, plan_t, a, b = case("f16", 64, 80, 60, [16, 5], 16, 3)
    bank = pp.AdapterBank(64, 80, 2, 16)
    bank.load_many([0, 1], a, b, p.c)
    want = outputs(p, bank, plan, plan_t)
    for slots, scales in (([1, 2], p.c), ([1, -1], p.c), ([1, 0], [1.0, float("nan")])):
        with pytest.raises(pp.PPError):
            bank.load_many(slots, a, b, scales)
    for wrong in (([a[0], a[1].float()], b), (a, [b[0], b[1].t()]), ([a[0], a[1][:, 1:]], b), ([a[0], a[1].cpu()], b), (a[:1], b), (a, [b[0], b[0]])):
        with pytest.raises(AssertionError):
            bank.load_many([0, 1], *wrong, p.c)
    with pytest.raises(AssertionError):
        bank.load_many([0], a, b, p.c)
    bank.load_many([], [], [], [])                                              # none to load
    for t, w in zip(outputs(p, bank, plan, plan_t), want):
        assert torch.equal(t, w)


def test_captured_loads_replay_with_other_weights():
    """The list is read when the call is made, the matrices when the graph runs."""
    ranks = [4 + i % 9 for i in range(70)]
    p, plan, plan_t, a, b = case("f16", 96, 64, 140, ranks, 12, 4)
    bank, other = pp.AdapterBank(96, 64, 70, 12), pp.AdapterBank(96, 64, 70, 12)
    x, slot_of = dev(p.x), dev(p.slot_of)
    bank.load_many(range(70), a, b, p.c)
    bank.run(plan, x, slot_of)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bank.load_many(range(70), a, b, p.c)
        y = bank.run(plan, x, slot_of)
    for i in range(4):
        for t in a:
            t.mul_(0.75)
        for s in range(70):
            other.load(s, a[s], b[s], p.c[s])
        want = other.run(plan, x, slot_of)
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


def test_on_a_stream_of_its_own():
    p, plan, plan_t, a, b = case("f32", 40, 33, 50, [8, 3, 5], 8, 5)
    bank, other = pp.AdapterBank(40, 33, 3, 8, pp.PP_F32), pp.AdapterBank(40, 33, 3, 8, pp.PP_F32)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    bank.load_many([0, 1, 2], a, b, p.c, stream=stream.cuda_stream)
    stream.synchronize()
    for s in range(3):
        other.load(s, a[s], b[s], p.c[s])
    for t, w in zip(outputs(p, bank, plan, plan_t), outputs(p, other, plan, plan_t)):
        assert torch.equal(t, w)
