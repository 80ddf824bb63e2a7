"""Host-side tests of the adapters, the 8-bit activations and transposed plans (no GPU): refusals, sizes, packing, symbols."""
import ctypes
import os
import re

import numpy as np
import pytest

import synth
import paper_2206_10620_amd as pp
from adapter_util import held8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
H = pp.PP_FLAG_HOST_ONLY
M32 = 1 << 20                    # addresses far enough apart; a host-only bank touches none


def bank(m=64, k=32, slots=4, max_rank=8, dtype=pp.PP_F16, flags=H):
    return pp.pp_adapter_plan(m, k, slots, max_rank, dtype, flags)


def test_bank_refusals():
    for bad in (dict(m=0), dict(k=0), dict(m=1 << 16, k=1 << 15), dict(slots=0), dict(slots=65537), dict(max_rank=0), dict(max_rank=129),
                dict(m=(1 << 22) + 1, k=1), dict(m=1, k=(1 << 22) + 1)):
        assert bank(**bad)[0] == pp.PP_ERR_SHAPE, bad
    assert bank(dtype=2)[0] == pp.PP_ERR_UNSUPPORTED
    assert bank(flags=H | pp.PP_FLAG_RELU)[0] == pp.PP_ERR_UNSUPPORTED
    assert pp.lib().pp_adapter_plan(None, None) == pp.PP_ERR_NULL
    assert pp.pp_adapter_destroy(None) == pp.PP_OK


@pytest.fixture
def small():
    st, h = bank()
    assert st == pp.PP_OK
    lay = synth.random_block_layer("a", 64, 32, 8, 16, 16, "f16", 0.5, 0.5, 3)
    plan, plan_t = pp.block_plan_from_layer(lay, host_only=True), pp.block_plan_transposed_from_layer(lay, host_only=True)
    yield h, plan, plan_t
    plan.close()
    plan_t.close()
    pp.pp_adapter_destroy(h)


def test_load_refusals(small):
    h = small[0]
    assert pp.pp_adapter_load(None, 0, 1, 1.0, 16, 32) == pp.PP_ERR_NULL
    assert pp.pp_adapter_load(h, 0, 1, 1.0, 0, 32) == pp.PP_ERR_NULL
    assert pp.pp_adapter_load(h, 0, 1, 1.0, 16, 0) == pp.PP_ERR_NULL
    for slot, rank in ((-1, 1), (4, 1), (0, -1), (0, 9)):
        assert pp.pp_adapter_load(h, slot, rank, 1.0, 16, 32) == pp.PP_ERR_SHAPE
    for scale in (float("inf"), float("-inf"), float("nan")):
        assert pp.pp_adapter_load(h, 0, 1, scale, 16, 32) == pp.PP_ERR_UNSUPPORTED
    assert pp.pp_adapter_load(h, 0, 1, 1.0, 18, 32) == pp.PP_ERR_ALIGN
    assert pp.pp_adapter_load(h, 0, 1, 1.0, 16, 40) == pp.PP_ERR_ALIGN
    assert pp.pp_adapter_load(h, 0, 0, 1.0, 0, 0) == pp.PP_ERR_UNSUPPORTED         # all in order, but the bank is host-only


def test_run_refusals(small):
    h, plan, plan_t = small
    a = [M32 * i for i in range(1, 9)]
    run = lambda **kw: pp.pp_adapter_run(*{**dict(bank=h, plan=plan.handle, x=a[0], s=a[1], u=a[2], y=a[3], n=8), **kw}.values())
    for name in ("bank", "plan", "x", "s", "u", "y"):
        assert run(**{name: None}) == pp.PP_ERR_NULL, name
    for n in (0, -1, (1 << 22) + 1):
        assert run(n=n) == pp.PP_ERR_SHAPE
    for name in ("x", "u", "y"):
        assert run(**{name: a[7] + 8}) == pp.PP_ERR_ALIGN, name
    assert run(y=a[0]) == run(y=a[0] + 16) == run(u=a[0]) == run(u=a[1]) == run(y=a[1]) == run(u=a[3]) == pp.PP_ERR_ALIGN
    assert run(s=a[7] + 2) == pp.PP_ERR_ALIGN
    assert run(plan=plan_t.handle) == pp.PP_ERR_SHAPE
    assert run(s=a[7] + 4) == run() == pp.PP_ERR_UNSUPPORTED
    other = synth.random_block_layer("a", 64, 32, 8, 16, 16, "f32", 0.5, 0.5, 3)
    p32 = pp.block_plan_from_layer(other, host_only=True)
    assert run(plan=p32.handle) == pp.PP_ERR_UNSUPPORTED                           # another storage type
    p32.close()
    project = lambda **kw: pp.pp_adapter_project(*{**dict(bank=h, x=a[0], s=a[1], u=a[2], n=8), **kw}.values())
    for name in ("bank", "x", "s", "u"):
        assert project(**{name: None}) == pp.PP_ERR_NULL, name
    assert project(n=0) == pp.PP_ERR_SHAPE and project(s=a[1] + 1) == project(u=a[0]) == project(x=a[0] + 2) == pp.PP_ERR_ALIGN and project() == pp.PP_ERR_UNSUPPORTED


def test_gradient_refusals(small):
    h, plan, plan_t = small
    a = [M32 * i for i in range(1, 14)]
    gi = lambda **kw: pp.pp_adapter_grad_input(*{**dict(bank=h, plan=plan_t.handle, dy=a[0], gate=a[1], g=a[2], s=a[3], v=a[4], dx=a[5], n=8), **kw}.values())
    for name in ("bank", "plan", "dy", "g", "s", "v"):
        assert gi(**{name: None}) == pp.PP_ERR_NULL, name
    assert gi(n=0) == pp.PP_ERR_SHAPE and gi(plan=plan.handle) == pp.PP_ERR_SHAPE
    for name in ("dy", "gate", "g", "v", "dx"):
        assert gi(**{name: a[9] + 4}) == pp.PP_ERR_ALIGN, name
    for kw in (dict(v=a[0]), dict(v=a[1]), dict(v=a[2]), dict(dx=a[0]), dict(dx=a[1]), dict(dx=a[2]), dict(dx=a[4]), dict(g=a[0] + 16), dict(g=a[1]), dict(v=a[3]), dict(dx=a[3])):
        assert gi(**kw) == pp.PP_ERR_ALIGN, kw
    assert gi(s=a[3] + 2) == pp.PP_ERR_ALIGN
    # in place, without a gate, without dx: in order but for the host-only bank
    assert gi(g=a[0]) == gi(gate=None, g=None) == gi(plan=None, dx=None) == pp.PP_ERR_UNSUPPORTED
    gw = lambda **kw: pp.pp_adapter_grad_weights(*{**dict(bank=h, x=a[0], held=0, u=a[1], g=a[2], v=a[3], s=a[4], which=a[5], count=2, da=a[6], db=a[7], work=a[8],
                                                          n=8), **kw}.values())
    for name in ("bank", "x", "u", "g", "v", "s", "which", "da", "db", "work"):
        assert gw(**{name: None}) == pp.PP_ERR_NULL, name
    assert gw(n=0) == gw(count=0) == gw(count=65536) == pp.PP_ERR_SHAPE
    for name in ("x", "u", "g", "v", "da", "db", "work"):
        assert gw(**{name: a[9] + 8}) == pp.PP_ERR_ALIGN, name
    for out in ("da", "db", "work"):
        for other in range(6):
            assert gw(**{out: a[other]}) == pp.PP_ERR_ALIGN, (out, other)
    assert gw(s=a[4] + 2) == gw(which=a[5] + 1) == pp.PP_ERR_ALIGN
    assert gw(db=a[6]) == gw(work=a[7]) == pp.PP_ERR_ALIGN
    assert gw() == gw(held=1) == pp.PP_ERR_UNSUPPORTED


def test_sizes(small):
    h = small[0]
    for f in (pp.pp_adapter_u_bytes, pp.pp_adapter_v_bytes):
        assert f(None, 8) == f(h, 0) == f(h, (1 << 22) + 1) == 0
        assert all(f(h, n) % 16 == 0 and f(h, n) >= n * 16 * 4 for n in (1, 7, 100, 5000))
    assert pp.pp_adapter_work_bytes(h, 8, 0) == pp.pp_adapter_work_bytes(h, 0, 1) == pp.pp_adapter_work_bytes(None, 8, 1) == 0
    assert pp.pp_adapter_work_bytes(h, 8, 1) >= 16
    assert pp.pp_act8_bytes(0, 8) == pp.pp_act8_bytes(8, 0) == pp.pp_act8_bytes(1 << 16, 1 << 15) == 0
    assert pp.pp_act8_bytes(3, 1) == 3 * 128 + 16 and pp.pp_act8_bytes(17, 300) == 17 * 384 + 3 * 32


def test_act8_refusals():
    for f in (pp.pp_act8_pack, lambda x, r, n, d, h: pp.pp_act8_unpack(h, r, n, d, x)):
        assert f(None, 4, 4, pp.PP_F16, 4096) == f(4096, 4, 4, pp.PP_F16, None) == pp.PP_ERR_NULL
        assert f(4096, 0, 4, pp.PP_F16, 8192) == f(4096, 4, 0, pp.PP_F16, 8192) == f(4096, 1 << 16, 1 << 15, pp.PP_F16, 8192) == pp.PP_ERR_SHAPE
        assert f(4096, 4, 4, 2, 8192) == pp.PP_ERR_UNSUPPORTED
        assert f(4096 + 2, 4, 4, pp.PP_F16, 8192) == f(4096, 4, 4, pp.PP_F16, 8192 + 8) == f(4096, 4, 4, pp.PP_F16, 4096 + 16) == pp.PP_ERR_ALIGN


@pytest.mark.parametrize("shape", [(130, 200, 50, 70), (64, 64, 64, 64), (33, 7, 4, 3), (1, 100, 8, 16)], ids=str)
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_transposed_plan_holds_the_transposed_weights(dtype, shape):
    m, k, bm, bk = shape
    lay = synth.random_block_layer("t", m, k, 8, bm, bk, dtype, 0.6, 0.5, seed=m + k, relu=True)
    want = np.where(lay.keep_matrix(), lay.weights.astype(np.float16 if dtype == "f16" else np.float32).astype(np.float32), 0.0).T
    plan = pp.block_plan_transposed_from_layer(lay, host_only=True)
    q = plan.query()
    assert (q["m"], q["k"], q["block_m"], q["block_k"]) == (k, m, bk, bm) and (plan.m, plan.k) == (k, m)
    assert q["kept_weights"] == lay.kept_weights
    for t in range(q["row_tiles"]):
        st, tile = pp.pp_block_gemm_unpack(plan.handle, t, 64, m)
        rows = min(64, k - 64 * t)
        assert st == pp.PP_OK and np.array_equal(tile[:rows], want[64 * t: 64 * t + rows]) and not tile[rows:].any()
    plan.close()


def test_transposed_plan_refusals():
    lay = synth.random_block_layer("t", 64, 32, 8, 16, 16, "f16", 0.5, 0.5, 1)
    args = lambda **kw: {**dict(m=64, k=32, block_m=16, block_k=16, row_keep=lay.row_keep, col_keep=lay.col_keep, weights=lay.weights, flags=H), **kw}
    f = pp.pp_block_gemm_plan_transposed
    assert f(**args(weights=None))[0] == pp.PP_ERR_NULL
    assert f(**args(m=0))[0] == f(**args(k=0))[0] == f(**args(block_m=0))[0] == pp.PP_ERR_SHAPE
    assert f(**args(flags=H | 64))[0] == f(**args(dtype=7))[0] == f(**args(variant=3))[0] == pp.PP_ERR_UNSUPPORTED
    st, h = f(**args(row_keep=None, col_keep=None))
    assert st == pp.PP_OK and pp.pp_block_gemm_query(h)[1]["kept_weights"] == 64 * 32
    pp.pp_block_gemm_destroy(h)


def test_the_8_bit_form_by_hand():
    """The reference that the GPU tests compare with, on values worked out by hand."""
    x = np.array([[127.0, 0.49, -0.5, 1.5, 2.5, 0.0, -126.6], [127.1, 0.9, 1.0, 3.0, -0.01, 5.0, 0.0]])
    assert held8(x).tolist() == [[127, 1, -1, 2, 2, 0, -127], [128, 2, 2, 4, -2, 4, 0]]
    assert held8(np.array([[0.0, -0.0]])).tolist() == [[0, 0]] and np.isnan(held8(np.array([[1.0, np.inf]]))).all()


def test_library_exports_every_declared_symbol():
    lib = ctypes.CDLL(pp.library_path())
    found = set()
    for header, pattern in (("pp_adapter.h", r"\b(pp_adapter_[a-z0-9_]+)\s*\("), ("pp_act8.h", r"\b(pp_act8_[a-z0-9_]+)\s*\(")):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        found |= set(re.findall(pattern, text))
    assert {"pp_adapter_plan", "pp_adapter_run", "pp_adapter_grad_weights", "pp_act8_pack", "pp_act8_unpack"} <= found
    for name in found | {"pp_block_gemm_plan_transposed"}:
        assert hasattr(lib, name), name
        assert hasattr(pp, name), name
