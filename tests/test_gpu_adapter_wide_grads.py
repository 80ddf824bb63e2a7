"""Gradients of layers so large that a wavefront takes two row tiles, in every form: binary16 and binary32, x as it is and in 8 bits.
The reference is the formula in 64 bits on the GPU, within the bounds of adapter_util."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m,k,n,ranks", [(4096, 4096, 4096, [64, 40]), (4090, 4083, 4101, [33, 48]), (2061, 6100, 4219, [128, 100])], ids=str)
def test_two_row_tiles(m, k, n, ranks, dtype, held):
    print("case", m, k, n, ranks, dtype, held, flush=True)
    tdt, code = (torch.float16, pp.PP_F16) if dtype == "f16" else (torch.float32, pp.PP_F32)
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    x, dy = (normal(k, n) * torch.exp(normal(k, 1))).to(tdt), normal(m, n).to(tdt)
    a, b, c = [(normal(r, k) / k ** 0.5).to(tdt) for r in ranks], [(normal(m, r) / r ** 0.5).to(tdt) for r in ranks], [0.75, -1.5]
    most = max(ranks)
    bank = pp.AdapterBank(m, k, 2, most, code)
    bank.load_many([0, 1], a, b, c)
    slot_of = torch.randint(-1, 2, (n,), generator=gen, device="cuda", dtype=torch.int32)
    u = bank.project(x, slot_of)
    g = bank.grad_input(None, dy, slot_of)
    act8 = pp.act8_pack(x)
    da, db = bank.grad_weights(act8 if held else x, u, g.g, g.v, slot_of, torch.tensor([1, 0], dtype=torch.int32, device="cuda"))
    xs = (act8.unpack(pp.PP_F32) if held else x).double()
    for i, s in enumerate((1, 0)):
        t = (slot_of == s).nonzero().flatten()
        gt, xt, x0, a64, b64, r = dy[:, t].double(), xs[:, t].contiguous(), x[:, t].double(), a[s].double(), b[s].double(), ranks[s]
        v, low = b64.t().contiguous() @ gt, a64 @ x0
        v_size, low_size = b64.abs().t().contiguous() @ gt.abs(), a64.abs() @ x0.abs()
        want_a, room_a = c[s] * (v @ xt.t().contiguous()), abs(c[s]) * (v_size @ xt.abs().t().contiguous()) * (2 * m + 2 * n + 32) * 2.0 ** -24
        want_b, room_b = c[s] * (gt @ low.t().contiguous()), abs(c[s]) * (gt.abs() @ low_size.t().contiguous()) * (2 * k + 2 * n + 32) * 2.0 ** -24
        assert bool(((da[i, :r].double() - want_a).abs() <= room_a).all()), "dA"
        assert bool(((db[i, :, :r].double() - want_b).abs() <= room_b).all()), "dB"
        assert not da[i, r:].any() and not db[i, :, r:].any()
        # far closer than the bound: binary32 sums of values of two binary16 parts or of binary32
        for got, want, what in ((da[i, :r], want_a, "dA"), (db[i, :, :r], want_b, "dB")):
            print(what, "relative to the largest", float((got.double() - want).abs().max() / want.abs().max()), flush=True)
    again = bank.grad_weights(act8 if held else x, u, g.g, g.v, slot_of, torch.tensor([1, 0], dtype=torch.int32, device="cuda"))
    assert torch.equal(da, again[0]) and torch.equal(db, again[1])
