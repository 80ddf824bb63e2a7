"""The adapters on the GPU against the formulas in 64 bits, within bounds that count roundings."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import Problem, assert_within, held8

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make_bank(p):
    bank = pp.AdapterBank(p.m, p.k, p.slots, p.max_rank, pp.PP_F16 if p.dtype == "f16" else pp.PP_F32)
    for s, r in enumerate(p.ranks):
        if r:
            bank.load(s, dev(p.a[s]), dev(p.b[s]), p.c[s])
    return bank


class Setup:
    def __init__(self, p):
        print(f"case {p.dtype} m={p.m} k={p.k} n={p.n} ranks={p.ranks[:6]} max_rank={p.max_rank} relu={p.relu}", flush=True)
        self.p = p
        self.bank = make_bank(p)
        self.plan, self.plan_t = pp.block_plan_from_layer(p.layer), pp.block_plan_transposed_from_layer(p.layer)
        self.x, self.dy, self.slot_of = dev(p.x), dev(p.dy), dev(p.slot_of)

    def check_forward(self):
        y, bound = self.p.forward()
        assert_within(self.bank.run(self.plan, self.x, self.slot_of).cpu().numpy(), y, bound, "y")

    def step(self, held=False, gate=None, which=None, plan_t=True):
        which = list(range(self.p.slots)) if which is None else which
        u = self.bank.project(self.x, self.slot_of)
        x = pp.act8_pack(self.x) if held else self.x
        g = self.bank.grad_input(self.plan_t if plan_t else None, self.dy, self.slot_of, gate=gate)
        da, db = self.bank.grad_weights(x, u, g.g, g.v, self.slot_of, dev(np.array(which, np.int32)))
        return g, da, db

    def check_backward(self, held=False, relu=False, which=None):
        p = self.p
        which = list(range(p.slots)) if which is None else which
        y = np.maximum(np.random.RandomState(5).standard_normal((p.m, p.n)), 0).astype(p.dy.dtype)
        g, da, db = self.step(held, pp.act8_pack(dev(y)) if relu else None, which)
        want, bounds = p.backward(held8(p.x) if held else p.x, y > 0 if relu else None, which)
        assert_within(g.dx.cpu().numpy(), want[0], bounds[0], "dx")
        assert_within(da.cpu().numpy(), want[1], bounds[1], "dA")
        assert_within(db.cpu().numpy(), want[2], bounds[2], "dB")
        if relu:
            assert np.array_equal(g.g.cpu().numpy(), np.where(y > 0, p.dy, 0).astype(p.dy.dtype))


# m, k, n, ranks, max_rank, order
SHAPES = [
    (64, 64, 1, [16], 16, "one"),                        # one token
    (130, 100, 2, [1, 5], 8, "mixed"),
    (64, 31, 7, [3], 3, "one"),                          # fewer rows than a step
    (1, 1, 1, [1], 1, "one"),
    (70, 200, 33, [16, 17, 0, 64], 64, "values"),        # an empty slot, entries that are no slot
    (256, 520, 64, list(range(1, 65)), 64, "mixed"),     # a rank and a slot to a token
    (100, 96, 100, [128, 128, 65], 128, "runs"),         # the largest rank
    (65, 129, 129, [8, 8], 24, "none"),
    (96, 333, 260, [4, 20], 32, "runs"),                 # two tokens to a lane
    (200, 64, 1030, [16, 16, 16], 16, "runs"),           # four tokens to a lane
    (64, 72, 2051, [32, 48], 48, "mixed"),
]


@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s[:3]) + s[5])
def test_forward(shape, dtype, relu):
    m, k, n, ranks, max_rank, order = shape
    Setup(Problem(dtype, m, k, n, ranks, max_rank, order, relu=relu, seed=m + n)).check_forward()


@pytest.mark.parametrize("held,relu", [(False, False), (True, True)])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s[:3]) + s[5])
def test_backward(shape, dtype, held, relu):
    m, k, n, ranks, max_rank, order = shape
    Setup(Problem(dtype, m, k, n, ranks, max_rank, order, seed=m + n)).check_backward(held, relu)


@pytest.mark.parametrize("n", [4096, 4101])
def test_many_columns(n):
    """The 512-column tile of the block product, whole and with rows that are no multiple of 16 bytes."""
    s = Setup(Problem("f16", 1024, 256, n, [16, 40], 40, "runs", relu=True, bm=64, bk=64, seed=n))
    s.check_forward()
    s = Setup(Problem("f16", 256, 1024, n, [16, 40], 40, "mixed", bm=64, bk=64, seed=n))
    s.check_backward(True, True)


def test_listed_slots():
    """Slots in any order, twice, ones that no token names, empty ones, numbers that are no slot."""
    p = Problem("f16", 96, 80, 300, [8, 16, 0, 4], 16, "runs", seed=3)
    p.slot_of[p.slot_of == 3] = 1
    Setup(p).check_backward(which=[1, 0, 1, 2, 3, -1, 4, 2 ** 31 - 1])


def test_no_gradient_for_x():
    p = Problem("f32", 48, 80, 200, [8, 16], 16, "runs", seed=4)
    s = Setup(p)
    g, da, db = s.step(plan_t=False)
    g2, da2, db2 = s.step()
    assert g.dx is None and torch.equal(da, da2) and torch.equal(db, db2)


def test_large_and_small_numbers():
    """u far beyond binary16 in a binary16 bank, and far below; y is not."""
    p = Problem("f16", 64, 512, 70, [16, 40], 40, "runs", seed=6)
    p.a = [(np.sign(a.astype(np.float32)) * 3e4).astype(np.float16) for a in p.a]
    p.b = [(b.astype(np.float32) * 2.0 ** -10).astype(np.float16) for b in p.b]
    p.x = (np.sign(p.x.astype(np.float32)) * 100).astype(np.float16)
    p.c = [2.0 ** -12, 2.0 ** -13]
    s = Setup(p)
    s.check_forward()
    s.check_backward()
    p.x[:, 1::2] = (p.x[:, 1::2].astype(np.float32) * 2.0 ** -20).astype(np.float16)     # small tokens beside large ones
    s = Setup(p)
    s.check_forward()
    s.check_backward()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_infinities_and_nan_stay_where_they_are(dtype):
    """A NaN in one token and an infinity in one slot's matrices reach that token, that slot's tokens and gradients, nothing else."""
    p = Problem(dtype, 80, 96, 200, [16, 24, 5], 24, "mixed", seed=7)
    clean = Setup(p)
    y0 = clean.bank.run(clean.plan, clean.x, clean.slot_of)
    g0, da0, db0 = clean.step()
    spoilt = int(np.flatnonzero(p.slot_of == 2)[0])
    p.x[3, spoilt] = np.nan
    p.dy[5, spoilt] = np.inf
    p.a[1][2, 7], p.b[1][9, 3] = np.inf, np.nan
    s = Setup(p)
    y = s.bank.run(s.plan, s.x, s.slot_of)
    g, da, db = s.step()
    good = torch.from_numpy(np.flatnonzero((p.slot_of != 1) & (np.arange(p.n) != spoilt))).cuda()
    assert torch.equal(y[:, good], y0[:, good]) and torch.equal(g.dx[:, good], g0.dx[:, good])
    assert torch.equal(da[0], da0[0]) and torch.equal(db[0], db0[0])
    assert not torch.isfinite(y[:, spoilt]).any() and not torch.isfinite(da[2, :5]).all()
    assert not torch.isfinite(y[9, torch.from_numpy(p.slot_of == 1).cuda()]).any()


def test_a_block_that_stands_for_nan():
    p = Problem("f16", 64, 48, 300, [8, 8], 8, "runs", seed=8)
    p.slot_of[:] = 0
    p.slot_of[128:] = 1
    s = Setup(p)
    x = p.x.copy()
    x[4, 10] = np.inf
    held = pp.act8_pack(dev(x))
    g = s.bank.grad_input(None, s.dy, s.slot_of)
    u = s.bank.project(s.x, s.slot_of)
    which = dev(np.array([0, 1], np.int32))
    da, db = s.bank.grad_weights(held, u, g.g, g.v, s.slot_of, which)
    da0, db0 = s.bank.grad_weights(pp.act8_pack(s.x), u, g.g, g.v, s.slot_of, which)
    assert torch.isnan(da[0, :, 4]).all() and torch.equal(da[1], da0[1]) and torch.equal(db, db0)
    keep = torch.arange(p.k, device="cuda") != 4
    assert torch.equal(da[0][:, keep], da0[0][:, keep])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_loading_again_and_unloading(dtype):
    p = Problem(dtype, 64, 80, 100, [16, 4], 32, "runs", seed=9)
    s = Setup(p)
    rs = np.random.RandomState(1)
    p.ranks[0], p.c[0] = 30, 0.5                                       # another rank in the same slot
    p.a[0], p.b[0] = rs.standard_normal((30, 80)).astype(p.x.dtype), rs.standard_normal((64, 30)).astype(p.x.dtype)
    s.bank.load(0, dev(p.a[0]), dev(p.b[0]), p.c[0])
    s.check_forward()
    s.check_backward()
    p.ranks[0] = 3                                                     # a smaller one: nothing is left of the larger
    p.a[0], p.b[0] = p.a[0][:3].copy(), p.b[0][:, :3].copy()
    s.bank.load(0, dev(p.a[0]), dev(p.b[0]), p.c[0])
    s.check_forward()
    s.check_backward()
    s.bank.unload(0)
    p.ranks[0], p.a[0], p.b[0] = 0, p.a[0][:0], p.b[0][:, :0]
    s.check_forward()
    s.check_backward()


def test_without_adapters_it_is_the_block_product():
    for dtype in ("f16", "f32"):
        p = Problem(dtype, 130, 200, 77, [16], 16, "none", relu=True, seed=10)
        s = Setup(p)
        assert torch.equal(s.bank.run(s.plan, s.x, s.slot_of), s.plan.run(s.x))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("keep", [0.0, 1.0])
def test_nothing_and_all_of_the_layer_kept(dtype, keep):
    """Empty column lists: the bias and the adapters alone; and a layer without a pruned weight."""
    for n in (3, 130):
        s = Setup(Problem(dtype, 100, 72, n, [16, 33], 40, "mixed", relu=True, keep=keep, seed=17))
        s.check_forward()
        s.check_backward(True, True)
    s = Setup(Problem(dtype, 4096, 64, 4096, [4], 4, "runs", keep=keep, bm=64, bk=64, seed=18))       # the 512-column tile
    s.check_forward()


def test_padding_tokens_may_hold_anything():
    """Tokens without an adapter, as a padded batch has them, filled with NaN and infinities: the others and all gradients are untouched."""
    p = Problem("f16", 96, 130, 400, [16, 24], 24, "mixed", seed=19)
    s = Setup(p)
    y0 = s.bank.run(s.plan, s.x, s.slot_of)
    g0, da0, db0 = s.step(held=True)
    pad = p.slot_of < 0
    p.x[:, pad], p.dy[:, pad] = np.nan, np.inf
    s2 = Setup(p)
    y = s2.bank.run(s2.plan, s2.x, s2.slot_of)
    u = s2.bank.project(s2.x, s2.slot_of)
    g = s2.bank.grad_input(s2.plan_t, s2.dy, s2.slot_of)
    da, db = s2.bank.grad_weights(s2.x, u, g.g, g.v, s2.slot_of, dev(np.array([0, 1], np.int32)))
    keep = torch.from_numpy(np.flatnonzero(~pad)).cuda()
    _, da1, db1 = s.step()
    assert torch.equal(y[:, keep], y0[:, keep]) and torch.equal(g.dx[:, keep], g0.dx[:, keep])
    assert torch.equal(da, da1) and torch.equal(db, db1) and torch.equal(db, db0) and torch.isfinite(da0).all()


@pytest.mark.parametrize("scale", [0.0, -1.5, 1e-30, 3e38])
def test_factors(scale):
    """A factor of zero, a negative one, the ends of binary32; with the largest B is zero, and so is the part it stands before."""
    p = Problem("f32" if scale == 1e-30 else "f16", 64, 48, 40, [8], 8, "one", seed=20)
    p.c[0] = float(np.float32(scale))
    if scale > 1:
        p.b[0][:] = 0
    s = Setup(p)
    s.check_forward()
    if scale <= 1:
        s.check_backward()


def _far(dtype, k, n, m, last):
    """A product whose x passes 2^32 bytes, adapters on its first and last tokens only; the reference takes those tokens alone."""
    tdt = torch.float16 if dtype == "f16" else torch.float32
    lay = Problem(dtype, m, k, 1, [8], 8, seed=21).layer
    plan = pp.block_plan_from_layer(lay)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((k, n), dtype=tdt, device="cuda")
    for r in range(0, k, 64):
        x[r:r + 64] = torch.randn((min(64, k - r), n), generator=gen, device="cuda").to(tdt)
    slot_of = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    slot_of[:5] = 0
    slot_of[n - last:] = 0
    a, b = (torch.randn((8, k), generator=gen, device="cuda") / k ** 0.5).to(tdt), torch.randn((m, 8), generator=gen, device="cuda").to(tdt)
    bank = pp.AdapterBank(m, k, 1, 8, pp.PP_F16 if dtype == "f16" else pp.PP_F32)
    bank.load(0, a, b, 0.5)
    print("case far", dtype, k, n, flush=True)
    y, u = bank.run(plan, x, slot_of, keep=True)
    plain = plan.run(x)
    at = torch.cat([torch.arange(5), torch.arange(n - last, n)]).cuda()
    xs = x[:, at].double()
    wd = torch.from_numpy(np.where(lay.keep_matrix(), lay.weights, 0).astype(np.float32)).cuda().to(tdt).double()
    want = wd @ xs + torch.from_numpy(lay.bias).cuda().double()[:, None] + 0.5 * (b.double() @ (a.double() @ xs))
    size = wd.abs() @ xs.abs() + 0.5 * (b.abs().double() @ (a.abs().double() @ xs.abs())) + 1
    half = 2.0 ** -11 if dtype == "f16" else 2.0 ** -24
    assert bool(((y[:, at].double() - want).abs() <= half * want.abs() + (2 * k + 32) * 2.0 ** -24 * size).all())
    y[:, at] = plain[:, at]
    assert torch.equal(y, plain)
    dy = torch.ones((m, n), dtype=tdt, device="cuda")
    g = bank.grad_input(None, dy, slot_of)
    which = torch.zeros(1, dtype=torch.int32, device="cuda")
    da, db = bank.grad_weights(x, u, g.g, g.v, slot_of, which)
    v = b.double().sum(0)
    room = (2 * m + 2 * len(at) + 32) * 2.0 ** -24 * 0.5 * b.abs().double().sum(0)[:, None] * xs.abs().sum(1)[None]
    assert bool(((da[0].double() - 0.5 * v[:, None] * xs.sum(1)[None]).abs() <= room).all())
    us = a.double() @ xs
    room = (2 * k + 2 * len(at) + 32) * 2.0 ** -24 * 0.5 * (a.abs().double() @ xs.abs()).sum(1)[None]
    assert bool(((db[0].double() - 0.5 * us.sum(1)[None]).abs() <= room).all())
    plan.close()


def test_offsets_beyond_32_bits_f16():
    _far("f16", 500, (1 << 22) - 1, 8, 300)


def test_offsets_beyond_32_bits_f32():
    _far("f32", 260, 1 << 22, 8, 129)


def test_equal_calls_give_equal_bits():
    s = Setup(Problem("f16", 256, 512, 700, [16, 33], 40, "mixed", seed=11))
    a, b = s.step(), s.step()
    assert torch.equal(a[0].dx, b[0].dx) and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    assert torch.equal(s.bank.run(s.plan, s.x, s.slot_of), s.bank.run(s.plan, s.x, s.slot_of))


def test_nothing_is_written_behind_the_ends():
    p = Problem("f16", 67, 45, 131, [5, 9], 11, "runs", seed=12)
    s = Setup(p)
    L, h, stream = pp.lib(), s.bank.handle, torch.cuda.current_stream().cuda_stream
    held, gate = pp.act8_pack(s.x), pp.act8_pack(dev(np.abs(p.dy)))
    sizes = dict(u=pp.pp_adapter_u_bytes(h, p.n), v=pp.pp_adapter_v_bytes(h, p.n), work=pp.pp_adapter_work_bytes(h, p.n, 2), y=p.m * p.n * 2, g=p.m * p.n * 2,
                 dx=p.k * p.n * 2, da=2 * 11 * p.k * 4, db=2 * 11 * p.m * 4)
    buf = {name: torch.full((size + 512,), 99, dtype=torch.uint8, device="cuda") for name, size in sizes.items()}
    at = {name: b.data_ptr() for name, b in buf.items()}
    which = dev(np.array([1, 0], np.int32))
    assert pp.pp_adapter_run(h, s.plan.handle, s.x.data_ptr(), s.slot_of.data_ptr(), at["u"], at["y"], p.n, stream) == pp.PP_OK
    assert pp.pp_adapter_grad_input(h, s.plan_t.handle, s.dy.data_ptr(), gate.buffer.data_ptr(), at["g"], s.slot_of.data_ptr(), at["v"], at["dx"], p.n, stream) == pp.PP_OK
    assert pp.pp_adapter_grad_weights(h, held.buffer.data_ptr(), 1, at["u"], at["g"], at["v"], s.slot_of.data_ptr(), which.data_ptr(), 2, at["da"], at["db"],
                                      at["work"], p.n, stream) == pp.PP_OK
    for name, size in sizes.items():
        assert bool((buf[name][size:] == 99).all()), name
    assert L is not None


def test_captured_step_replays_with_other_tokens_and_weights():
    """A whole tuning step in a graph: loading, forward, 8-bit forms, both halves of the backward pass.  Each replay, with other
    contents in the same buffers and other work in between, gives what the eager calls give."""
    p = Problem("f16", 128, 192, 260, [16, 24], 24, "runs", relu=True, bm=32, bk=32, seed=13)
    s = Setup(p)
    a, b = dev(p.a[0]), dev(p.b[0])
    which = dev(np.array([0, 1], np.int32))

    def step():
        s.bank.load(0, a, b, p.c[0])
        y, u = s.bank.run(s.plan, s.x, s.slot_of, keep=True)
        g = s.bank.grad_input(s.plan_t, s.dy, s.slot_of, gate=pp.act8_pack(y))
        return (y, g.dx) + s.bank.grad_weights(pp.act8_pack(s.x), u, g.g, g.v, s.slot_of, which)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    rs = np.random.RandomState(2)
    for i in range(4):
        s.x.copy_(dev(rs.standard_normal(p.x.shape).astype(np.float16)))
        s.slot_of.copy_(dev(rs.randint(-1, 3, p.n).astype(np.int32)))
        a.mul_(0.5)
        want = [t.clone() for t in step()]
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(out, want):
            assert torch.equal(got, w), i


def test_two_streams_at_once():
    """Runs share the bank and the plan and nothing else."""
    p = Problem("f16", 256, 512, 300, [16, 33], 40, "mixed", relu=True, seed=14)
    s = Setup(p)
    x2 = (s.x * 0.5).contiguous()
    want, want2 = s.bank.run(s.plan, s.x, s.slot_of), s.bank.run(s.plan, x2, s.slot_of)
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    got, got2 = [], []
    for _ in range(10):
        got.append(s.bank.run(s.plan, s.x, s.slot_of, stream=one.cuda_stream))
        got2.append(s.bank.run(s.plan, x2, s.slot_of, stream=two.cuda_stream))
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for t in got) and all(torch.equal(t, want2) for t in got2)


def test_gradients_against_differences():
    """Binary32: the loss sum(w * y) moved along each gradient by central differences.  The loss is linear in A and in B apart from
    the ReLU, whose kinks are kept away by a large bias; what is left is rounding: 2^-24 of the loss's terms over the step."""
    p = Problem("f32", 40, 56, 90, [6, 3], 8, "runs", relu=True, seed=15)
    p.layer.bias[:] = np.where(np.arange(p.m) % 2 == 0, 100.0, -100.0).astype(np.float32)       # half of the rows open, half closed
    s = Setup(p)
    y = s.bank.run(s.plan, s.x, s.slot_of)
    g, da, db = s.step(gate=pp.act8_pack(y))
    rs = np.random.RandomState(3)

    def loss():
        return float((s.bank.run(s.plan, s.x, s.slot_of).double() * s.dy.double()).sum())

    room = 8 * 2.0 ** -24 * float((y.abs().double() * s.dy.abs().double()).sum())
    for slot in (0, 1):
        r = p.ranks[slot]
        for which, grad in (("a", da[slot, :r]), ("b", db[slot, :, :r])):
            move = rs.standard_normal(grad.shape).astype(np.float32)
            at, other = (p.a[slot], p.b[slot]) if which == "a" else (p.b[slot], p.a[slot])
            ends = []
            for sign in (1, -1):
                moved = dev(at + np.float32(sign) * move)
                s.bank.load(slot, *((moved, dev(other)) if which == "a" else (dev(other), moved)), p.c[slot])
                ends.append(loss())
            s.bank.load(slot, dev(p.a[slot]), dev(p.b[slot]), p.c[slot])
            want = float((grad.double().cpu() * torch.from_numpy(move).double()).sum())
            assert abs((ends[0] - ends[1]) / 2 - want) <= room, (slot, which, ends, want, room)
    move = dev(rs.standard_normal(p.x.shape).astype(np.float32))
    x0, ends = s.x.clone(), []
    for sign in (1, -1):
        s.x.copy_(x0 + sign * move)
        ends.append(loss())
    want = float((g.dx.double() * move.double()).sum())
    assert abs((ends[0] - ends[1]) / 2 - want) <= room, (ends, want, room)


def test_refusals_that_need_a_device():
    p = Problem("f16", 64, 64, 12, [8], 8, "one", seed=16)
    s = Setup(p)
    for variant in (1, 2):
        plan = pp.block_plan_from_layer(p.layer, variant=variant)
        with pytest.raises(pp.PPError) as e:
            s.bank.run(plan, s.x, s.slot_of)
        assert e.value.status == pp.PP_ERR_UNSUPPORTED
        plan.close()
    with pytest.raises(AssertionError):
        s.bank.run(s.plan, s.x.t(), s.slot_of)
    with pytest.raises(AssertionError):
        s.bank.run(s.plan, s.x, s.slot_of.long())
    s.bank.close()
    s.bank.close()
    for call in (lambda: s.bank.run(s.plan, s.x, s.slot_of), lambda: s.bank.project(s.x, s.slot_of), lambda: s.bank.unload(0),
                 lambda: s.bank.grad_input(s.plan_t, s.dy, s.slot_of)):
        with pytest.raises(pp.PPError) as e:
            call()
        assert e.value.status == pp.PP_ERR_NULL


def test_states_of_another_kind_are_refused():
    p = Problem("f16", 64, 80, 40, [8], 8, "one", seed=17)
    s = Setup(p)
    _, u = s.bank.run(s.plan, s.x, s.slot_of, keep=True)
    g = s.bank.grad_input(s.plan_t, s.dy, s.slot_of)
    which = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad_u, bad_v in ((u.cpu(), g.v), (u, g.v.cpu()), (u[1:], g.v), (u, g.v[:-1]), (torch.zeros(u.numel(), device="cuda"), g.v)):
        with pytest.raises(AssertionError):
            s.bank.grad_weights(s.x, bad_u, g.g, bad_v, s.slot_of, which)
    held = pp.act8_pack(s.x)
    for buffer, rows, n in ((held.buffer.cpu(), 80, 40), (held.buffer, 80, 129), (held.buffer[1:], 80, 40), (held.buffer, 0, 40), (s.x, 80, 40)):
        with pytest.raises(AssertionError):
            pp.Act8(buffer, rows, n, pp.PP_F16)
    da, db = s.bank.grad_weights(pp.Act8(held.buffer, 80, 40, pp.PP_F16), u, g.g, g.v, s.slot_of, which)
    assert da.shape == (1, 8, 80) and db.shape == (1, 64, 8)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("shape", [(130, 300, 513, [16, 3], 16, "runs"), (1056, 640, 545, [40, 64], 64, "mixed"), (96, 33, 1025, [20], 32, "one"),
                                   (544, 577, 2049, [16, 9, 12], 16, "runs"), (300, 129, 4097, [64, 33], 64, "runs"), (97, 256, 4223, [30, 0], 32, "values")],
                         ids=lambda s: "x".join(str(v) for v in s[:3]))
def test_tiles_of_several_tokens_to_a_lane(shape, dtype):
    """Token counts that end inside a tile, row counts that end inside a step, wavefronts with few and with many steps."""
    m, k, n, ranks, max_rank, order = shape
    for relu in (False, True):
        s = Setup(Problem(dtype, m, k, n, ranks, max_rank, order, relu=relu, seed=18))
        s.check_forward()
        s.check_backward(held=relu, relu=relu)
