"""Low-rank adapters beside the block-pruned product, their gradients, and activations held in 8 bits.

W is an m x k block-pruned matrix, x has one token per column, and every token names an adapter slot or none.  Slot s holds
A (rank x k), B (m x rank) and a factor c.  The kinds of cases are

  adapted     y = act(W x + bias + c B (A x)), every token with its own adapter: prompts, and single tokens of many requests
  gradient    what trains the adapters while W stays: dx = W^T g + c A^T (B^T g), dA = c (B^T g) x^T, dB = c g (A x)^T, with
              g = dy where the layer's output was positive if it had a ReLU; x, and the output for the ReLU, may be held in 8 bits
  checkpoint  x to 8 bits with a power of two for each row and 128 tokens, and back

`listed()` names the sizes, `draw()` takes others from the same ranges.
"""
from __future__ import annotations

import math
import types

import numpy as np
import torch

own = False

BLOCK8 = 128                                    # tokens that share a scale in the 8-bit form


# ---------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------

def _adapted(dtype, m, k, n, requests, slots, rank, rank_min=None, block=64, keep=0.41, relu=False, bare=False, load=False):
    return {"kind": "adapted", "dtype": dtype, "m": m, "k": k, "n": n, "requests": requests, "slots": slots, "rank": rank,
            "rank_min": rank_min or rank, "block": block, "keep": keep, "relu": relu, "bare": bare, "load": load}


def _gradient(dtype, m, k, n, requests, slots, rank, rank_min=None, block=64, keep=0.41, relu=False, bare=False, held="x"):
    return {"kind": "gradient", "dtype": dtype, "m": m, "k": k, "n": n, "requests": requests, "slots": slots, "rank": rank,
            "rank_min": rank_min or rank, "block": block, "keep": keep, "relu": relu, "bare": bare, "held": held}


def _checkpoint(dtype, k, n):
    return {"kind": "checkpoint", "dtype": dtype, "k": k, "n": n}


def listed():
    cases = [
        # one user's next token on a transformer's feed-forward projection: latency only
        ("adapted_f16_token", _adapted("f16", 4096, 4096, 1, 1, 1, 16)),
        # the next tokens of 64 users, each with an adapter of their own and of their own rank, some with none
        ("adapted_f16_64_users", _adapted("f16", 4096, 4096, 64, 64, 64, 64, 8, bare=True)),
        # prompts of several users in one odd batch of columns, sizes that fill no tile
        ("adapted_f16_ragged", _adapted("f16", 1775, 1023, 1003, 5, 4, 32, 8, block=16, keep=0.7, bare=True)),
        # a long batch of prompts
        ("adapted_f16_prompts", _adapted("f16", 4096, 4096, 4096, 8, 8, 32, relu=True)),
        # the forward pass of a tuning step: the adapters as the optimizer left them are loaded first
        ("adapted_f16_tuning", _adapted("f16", 4096, 1024, 2048, 1, 1, 16, relu=True, load=True)),
        # a classifier head in full precision
        ("adapted_f32_head", _adapted("f32", 1000, 2048, 197, 3, 3, 8, block=16, keep=0.7)),
        # the backward pass of a tuning step, activations held in 8 bits, the layer's ReLU undone
        ("gradient_f16_held8", _gradient("f16", 4096, 4096, 4096, 1, 1, 16, relu=True, held="act8")),
        # six adapters tuned at once on sequences of odd lengths, activations as they are
        ("gradient_f16_many", _gradient("f16", 1024, 4096, 2000, 7, 6, 64, 8, bare=True)),
        # the same in full precision on odd sizes, from 8 bits
        ("gradient_f32_odd", _gradient("f32", 777, 1023, 509, 3, 2, 24, 5, block=16, keep=0.7, relu=True, held="act8")),
        # the activations of a layer
        ("checkpoint_f16_4096", _checkpoint("f16", 4096, 4096)),
        # odd sizes in full precision
        ("checkpoint_f32_odd", _checkpoint("f32", 1023, 2051)),
        # the activations of one short sequence
        ("checkpoint_f16_small", _checkpoint("f16", 256, 100)),
    ]
    return [dict(case, name=name) for name, case in cases]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi] drawn evenly over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above; sizes over the logarithm, odd ones among them."""
    kind = rng.choice(["adapted", "adapted", "gradient", "gradient", "checkpoint"])
    dtype = rng.choice(["f16", "f16", "f32"])
    if kind == "checkpoint":
        return _checkpoint(dtype, _log_int(rng, 64, 4096), _log_int(rng, 16, 4096 if dtype == "f16" else 2048))
    top = 4096 if dtype == "f16" else 1024
    m, k = _log_int(rng, 64, top), _log_int(rng, 64, top)
    n = _log_int(rng, 1 if kind == "adapted" else 64, top)
    if rng.random() < 0.5:
        n = -(-n // 8) * 8
    requests = n if n <= 64 and rng.random() < 0.7 else rng.randint(1, min(n, 8))
    slots = rng.randint(1, min(requests, 64))
    rank = rng.choice([4, 8, 16, 16, 24, 32, 64, 128])
    common = dict(rank_min=max(1, rank // rng.choice([1, 2, 4])), block=rng.choice([16, 32, 64, 128]), keep=rng.choice([0.41, 0.7, 1.0]),
                  relu=rng.random() < 0.5, bare=rng.random() < 0.5)
    if kind == "adapted":
        return _adapted(dtype, m, k, n, requests, slots, rank, load=rng.random() < 0.2, **common)
    return _gradient(dtype, m, k, n, min(requests, 8), min(slots, 8), rank, held=rng.choice(["x", "act8"]), **common)


def _rank(case, slot):
    return max(case["rank_min"], case["rank"] // (1 + slot % 4))


def _slot(case, request):
    """The slot of a request; with `bare` every fifth request has no adapter."""
    return -1 if case["bare"] and request % 5 == 4 else request % case["slots"]


def work(case):
    eb = 2 if case["dtype"] == "f16" else 4
    k, n = case["k"], case["n"]
    if case["kind"] == "checkpoint":
        # x read, its 8-bit form written and read, the values written
        return {"bytes": k * n * (2 * eb + 2) + 2 * k * -(-n // BLOCK8), "flops": 4 * k * n}
    m = case["m"]
    kept = case["keep"] ** 2 * m * k
    used = sorted({_slot(case, r) for r in range(case["requests"])} - {-1})
    ranks = sum(_rank(case, s) for s in used)
    mean = ranks / max(1, len(used))
    if case["kind"] == "adapted":
        nbytes = (m + k) * n * eb + kept * eb + 4 * m + (m + k) * ranks * eb + 4 * n
        return {"bytes": int(nbytes), "flops": int(2 * n * (kept + (m + k) * mean))}
    x_bytes = k * n * (1 if case["held"] == "act8" else eb)
    gate = m * n if case["relu"] else 0
    nbytes = (m + k) * n * eb + kept * eb + x_bytes + gate + (m + k) * ranks * (eb + 4) + 4 * n * (mean + 1)
    return {"bytes": int(nbytes), "flops": int(2 * n * (kept + 2 * (m + k) * mean))}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _inputs(case, seed):
    """Everything a case is given, from the seed alone: tensors on the GPU, and the layer's description on the host."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tdt = torch.float16 if case["dtype"] == "f16" else torch.float32
    k, n = case["k"], case["n"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # features of a trained network differ in size: a factor of its own for each
    x = (normal(k, n) * torch.exp(0.7 * normal(k, 1))).to(tdt)
    if case["kind"] == "checkpoint":
        return types.SimpleNamespace(x=x, tdt=tdt)
    m, block = case["m"], case["block"]
    bm, bk = -(-m // block), -(-k // block)
    rs = np.random.RandomState(seed % (1 << 32))
    row_keep = (rs.random_sample((bm, bk, block)) < case["keep"]).astype(np.uint8)
    col_keep = (rs.random_sample((bm, bk, block)) < case["keep"]).astype(np.uint8)
    weights = normal(m, k) / math.sqrt(max(1.0, k * case["keep"] ** 2))
    bias = 0.01 * normal(m)
    # the requests' tokens stand one behind the other, at least one token each
    cuts = np.sort(rs.choice(n - 1, case["requests"] - 1, replace=False)) + 1 if case["requests"] > 1 else np.zeros(0, int)
    lengths = np.diff(np.concatenate([[0], cuts, [n]]))
    slots = np.array([_slot(case, r) for r in range(case["requests"])], np.int32)
    slot_of = np.repeat(slots, lengths)
    used = [int(s) for s in sorted(set(slots.tolist()) - {-1})]
    ranks = {s: _rank(case, s) for s in used}
    a = {s: (normal(ranks[s], k) / math.sqrt(k)).to(tdt) for s in used}
    b = {s: (0.5 * normal(m, ranks[s]) / math.sqrt(ranks[s])).to(tdt) for s in used}
    scale = {s: 2.0 / (1 + s % 3) for s in used}
    layer = types.SimpleNamespace(m=m, k=k, bm=block, bk=block, row_keep=row_keep, col_keep=col_keep, weights=weights.cpu().numpy(),
                                  bias=bias.cpu().numpy(), relu=case["relu"], dtype=case["dtype"])
    p = types.SimpleNamespace(x=x, tdt=tdt, layer=layer, bias=bias, slot_of=slot_of, used=used, ranks=ranks, a=a, b=b, scale=scale,
                              weights=weights.to(tdt))
    if case["kind"] == "gradient":
        p.dy = (0.1 * normal(m, n)).to(tdt)
        p.y = torch.clamp(normal(m, n), min=0.0).to(tdt)       # a ReLU's output: half of it zero
    return p


def _dense(layer, weights):
    """The pruned weights with zeros in their places."""
    rk = torch.from_numpy(layer.row_keep).cuda().bool()[:, :, :, None]
    ck = torch.from_numpy(layer.col_keep).cuda().bool()[:, :, None, :]
    keep = (rk & ck).permute(0, 2, 1, 3).reshape(rk.shape[0] * layer.bm, ck.shape[1] * layer.bk)[: layer.m, : layer.k]
    return torch.where(keep, weights, torch.zeros_like(weights))


def _groups(p):
    return [(s, torch.from_numpy(np.flatnonzero(p.slot_of == s)).cuda()) for s in p.used]


def prepare(case, seed):
    p = _inputs(case, seed)
    st = types.SimpleNamespace(case=case, x=p.x)
    if case["kind"] == "checkpoint":
        return st
    st.a, st.b, st.scale, st.used, st.ranks = p.a, p.b, p.scale, p.used, p.ranks
    st.slot_of = torch.from_numpy(p.slot_of).cuda()
    gradient = case["kind"] == "gradient"
    if own:
        import paper_2206_10620_amd as pp
        dtype = pp.PP_F16 if case["dtype"] == "f16" else pp.PP_F32
        st.bank = pp.AdapterBank(case["m"], case["k"], case["slots"], case["rank"], dtype)
        for s in p.used:
            st.bank.load(s, p.a[s], p.b[s], p.scale[s])
        if gradient:
            st.plan_t = pp.block_plan_transposed_from_layer(p.layer)
            st.u = st.bank.project(p.x, st.slot_of)            # what the forward pass left
            st.held = pp.act8_pack(p.x) if case["held"] == "act8" else p.x
            st.gate = pp.act8_pack(p.y) if case["relu"] else None
            st.which = torch.tensor(p.used, dtype=torch.int32, device="cuda")
            st.dy = p.dy
        else:
            st.plan = pp.block_plan_from_layer(p.layer)
        return st
    st.groups = _groups(p)
    st.weights = _dense(p.layer, p.weights)
    st.bias = p.bias
    if gradient:
        st.dy = p.dy
        st.positive = p.y > 0 if case["relu"] else None
        st.held = _pack(p.x) if case["held"] == "act8" else p.x
        st.u = {s: p.a[s].float() @ p.x[:, cols].float() for s, cols in st.groups}
    elif case["n"] <= 64 and p.used:
        # single tokens: the slots' matrices in one array, filled up with zeros, to be taken by index
        st.index = torch.clamp(st.slot_of, min=0).long()
        st.a_all = torch.zeros((case["slots"], case["rank"], case["k"]), dtype=p.tdt, device="cuda")
        st.b_all = torch.zeros((case["slots"], case["m"], case["rank"]), dtype=p.tdt, device="cuda")
        for s in p.used:
            st.a_all[s, : p.ranks[s]] = p.a[s]
            st.b_all[s, :, : p.ranks[s]] = p.b[s]
        factor = torch.tensor([p.scale.get(s, 0.0) for s in range(case["slots"])], device="cuda")
        st.factor = torch.where(st.slot_of >= 0, factor[st.index], torch.zeros_like(factor[st.index]))
    return st


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def run(state):
    kind = state.case["kind"]
    if own:
        return {"adapted": _run_adapted, "gradient": _run_gradient, "checkpoint": _run_checkpoint}[kind](state)
    return {"adapted": _plain_adapted, "gradient": _plain_gradient, "checkpoint": _plain_checkpoint}[kind](state)


def _run_adapted(st):
    if st.case["load"]:
        st.bank.load_many(st.used, [st.a[s] for s in st.used], [st.b[s] for s in st.used], [st.scale[s] for s in st.used])
    return st.bank.run(st.plan, st.x, st.slot_of)


def _run_gradient(st):
    grad = st.bank.grad_input(st.plan_t, st.dy, st.slot_of, gate=st.gate)
    da, db = st.bank.grad_weights(st.held, st.u, grad.g, grad.v, st.slot_of, st.which)
    return grad.dx, da, db


def _run_checkpoint(st):
    import paper_2206_10620_amd as pp
    return pp.act8_pack(st.x).unpack()


def _plain_adapted(st):
    c = st.case
    x = st.x.float()
    y = st.weights.float() @ x + st.bias[:, None]
    if c["n"] <= 64 and st.used:
        u = (st.a_all[st.index].float() * x.t()[:, None, :]).sum(2) * st.factor[:, None]
        y += (st.b_all[st.index].float() * u[:, None, :]).sum(2).t()
    else:
        for s, cols in st.groups:
            y[:, cols] += st.scale[s] * (st.b[s].float() @ (st.a[s].float() @ x[:, cols]))
    if c["relu"]:
        y = torch.clamp(y, min=0.0)
    return y.to(st.x.dtype)


def _plain_gradient(st):
    c = st.case
    g = st.dy.float()
    if st.positive is not None:
        g = torch.where(st.positive, g, torch.zeros_like(g))
    x = _unpack(*st.held, c["n"]) if c["held"] == "act8" else st.held.float()
    dx = st.weights.float().t() @ g
    da = torch.zeros((len(st.used), c["rank"], c["k"]), device="cuda")
    db = torch.zeros((len(st.used), c["m"], c["rank"]), device="cuda")
    for i, (s, cols) in enumerate(st.groups):
        gs = g[:, cols]
        v = st.scale[s] * (st.b[s].float().t() @ gs)
        dx[:, cols] += st.a[s].float().t() @ v
        da[i, : st.ranks[s]] = v @ x[:, cols].t()
        db[i, :, : st.ranks[s]] = st.scale[s] * (gs @ st.u[s].t())
    return dx.to(st.dy.dtype), da, db


def _pack(x):
    """x in 8 bits: whole numbers and, for every row and block of tokens, the power of two they are multiples of."""
    k, n = x.shape
    blocks = -(-n // BLOCK8)
    xf = torch.zeros((k, blocks * BLOCK8), device=x.device)
    xf[:, :n] = x
    xf = xf.view(k, blocks, BLOCK8)
    part, power = torch.frexp(xf.abs().amax(2, keepdim=True))                  # amax = part * 2^power, part in [0.5, 1)
    power = power - 7 + (part > 127.0 / 128.0).int()                           # the smallest with amax <= 127 * 2^power
    power = torch.clamp(power, min=-126)
    q = torch.round(torch.ldexp(xf, -power))
    q = torch.where(q == 0, torch.sign(xf), q)                                 # what is not zero stays so, with its sign
    return q.to(torch.int8), power


def _unpack(q, power, n):
    return torch.ldexp(q.float(), power).flatten(1)[:, :n]


def _plain_checkpoint(st):
    return _unpack(*_pack(st.x), st.case["n"]).to(st.x.dtype)


# ---------------------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def _held8_64(x):
    """What the 8-bit form of x stands for, value by value from its definition."""
    x = x.double()
    n = x.shape[1]
    out = torch.empty_like(x)
    for t in range(0, n, BLOCK8):
        part = x[:, t : t + BLOCK8]
        top = part.abs().amax(1, keepdim=True)
        step = torch.exp2(torch.clamp(torch.ceil(torch.log2(top / 127.0)), min=-126.0))
        step = torch.where(top > 127.0 * step, 2.0 * step, step)               # log2 may be off by its last bit
        step = torch.where(top <= 63.5 * step, torch.clamp(0.5 * step, min=2.0 ** -126), step)
        near = torch.round(part / step)
        near = torch.where((near == 0) & (part != 0), torch.sign(part), near)
        out[:, t : t + BLOCK8] = near * step
    return out


def exact(case, seed):
    p = _inputs(case, seed)
    if case["kind"] == "checkpoint":
        return _held8_64(p.x)
    slot_of = torch.from_numpy(p.slot_of).cuda()
    w = _dense(p.layer, p.weights).double()
    x = p.x.double()
    if case["kind"] == "adapted":
        y = w @ x + p.bias.double()[:, None]
        for s in p.used:
            mine = (slot_of == s).nonzero().flatten()
            low = p.a[s].double() @ x.index_select(1, mine)
            y.index_add_(1, mine, p.b[s].double() @ low, alpha=p.scale[s])
        return torch.relu(y) if case["relu"] else y
    g = p.dy.double()
    if case["relu"]:
        g = g * (p.y > 0).double()
    held = _held8_64(p.x) if case["held"] == "act8" else x
    dx = w.t() @ g
    da = torch.zeros((len(p.used), case["rank"], case["k"]), dtype=torch.float64, device="cuda")
    db = torch.zeros((len(p.used), case["m"], case["rank"]), dtype=torch.float64, device="cuda")
    for i, s in enumerate(p.used):
        mine = (slot_of == s).nonzero().flatten()
        gs = g.index_select(1, mine)
        low = p.a[s].double() @ x.index_select(1, mine)
        back = p.b[s].double().t() @ gs
        dx.index_add_(1, mine, p.a[s].double().t() @ back, alpha=p.scale[s])
        da[i, : p.ranks[s]] = p.scale[s] * (back @ held.index_select(1, mine).t())
        db[i, :, : p.ranks[s]] = p.scale[s] * (gs @ low.t())
    return dx, da, db
