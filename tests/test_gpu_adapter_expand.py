"""The binary32 adapters' part by both of its kernels: 16 tokens at a time, and 64, with many slots, every rank and odd sizes."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import Problem, assert_within

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Setup:
    def __init__(self, p):
        print("case", p.m, p.k, p.n, p.slots, p.max_rank, p.relu, flush=True)
        self.p = p
        self.bank = pp.AdapterBank(p.m, p.k, p.slots, p.max_rank, pp.PP_F32)
        some = [s for s in range(p.slots) if p.ranks[s]]
        self.bank.load_many(some, [dev(p.a[s]) for s in some], [dev(p.b[s]) for s in some], [p.c[s] for s in some])
        self.plan, self.plan_t = pp.block_plan_from_layer(p.layer), pp.block_plan_transposed_from_layer(p.layer)
        self.x, self.dy, self.slot_of = dev(p.x), dev(p.dy), dev(p.slot_of)

    def run(self):
        return self.bank.run(self.plan, self.x, self.slot_of), self.bank.grad_input(self.plan_t, self.dy, self.slot_of).dx


MANY = [1 + (5 * i) % 128 for i in range(60)]
# m, k, n, ranks, max_rank, order: workgroups of 16 x 16 at most 1024 (4096 with more than 16 slots), and more
SIZES = {
    "16 tokens, a slot each": (83, 60, 64, MANY, 128, "mixed"),
    "16 tokens, 9 ragged": (658, 65, 9, [128, 3, 17, 64, 0, 33], 128, "values"),
    "16 tokens, one row": (1, 40, 130, [20, 5], 32, "runs"),
    "16 tokens, one token": (1000, 33, 1, [16], 16, "one"),
    "16 tokens, all ranks of one slot": (130, 20, 33, [128], 128, "one"),
    "16 tokens, at the limit": (512, 48, 512, [8, 40], 40, "mixed"),
    "64 tokens, behind the limit": (513, 48, 512, [8, 40], 40, "mixed"),
    "16 tokens, many slots at the limit": (1024, 40, 1020, MANY, 128, "runs"),
    "64 tokens, many slots behind the limit": (1030, 40, 1030, MANY, 128, "mixed"),
    "64 tokens, ragged": (77, 50, 4099, [16, 100, 0, 1], 112, "values"),
}


@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("size", SIZES.values(), ids=SIZES.keys())
def test_against_the_formula(size, relu):
    m, k, n, ranks, max_rank, order = size
    p = Problem("f32", m, k, n, ranks, max_rank, order, relu=relu, seed=m + n)
    s = Setup(p)
    y, dx = s.run()
    want, bound = p.forward()
    assert_within(y.cpu().numpy(), want, bound, "y")
    wants, bounds = p.backward(p.x, None, [])
    assert_within(dx.cpu().numpy(), wants[0], bounds[0], "dx")
    again = s.run()
    assert torch.equal(y, again[0]) and torch.equal(dx, again[1])


@pytest.mark.parametrize("m,n", [(40, 50), (600, 1100)], ids=str)
def test_what_is_no_number_stays_with_its_tokens(m, n):
    """A slot's infinities, a token's NaN, and columns of tokens that have no adapter."""
    p = Problem("f32", m, 48, n, [16, 40, 5], 40, "mixed", seed=50)
    clean = Setup(p)
    y0 = clean.run()[0]
    plain = clean.plan.run(clean.x)
    none = dev(np.flatnonzero(p.slot_of < 0))
    assert torch.equal(y0[:, none], plain[:, none])
    spoilt = int(np.flatnonzero(p.slot_of == 2)[0])
    p.x[3, spoilt] = np.nan
    p.a[1][2, 7], p.b[1][m - 1, 3] = np.inf, np.nan
    y = Setup(p).run()[0]
    good = dev(np.flatnonzero((p.slot_of != 1) & (np.arange(n) != spoilt)))
    assert torch.equal(y[:, good], y0[:, good])
    assert torch.isnan(y[:, spoilt]).all() and not torch.isfinite(y[:, dev(np.flatnonzero(p.slot_of == 1))]).any()


@pytest.mark.parametrize("m,n", [(37, 45), (600, 1100)], ids=str)
def test_nothing_is_written_behind_the_end(m, n):
    p = Problem("f32", m, 20, n, [5, 18], 32, "mixed", seed=51)
    s = Setup(p)
    u = torch.full((pp.pp_adapter_u_bytes(s.bank.handle, n) + 256,), 255, dtype=torch.uint8, device="cuda")       # NaN where nothing is written
    y = torch.full((m * n + 64,), 7.0, device="cuda")
    assert pp.pp_adapter_run(s.bank.handle, s.plan.handle, s.x.data_ptr(), s.slot_of.data_ptr(), u.data_ptr(), y.data_ptr(), n,
                             torch.cuda.current_stream().cuda_stream) == pp.PP_OK
    assert bool((y[m * n:] == 7.0).all()) and bool((u[-256:] == 255).all())
    want, bound = p.forward()
    assert_within(y[: m * n].view(m, n).cpu().numpy(), want, bound, "y")
