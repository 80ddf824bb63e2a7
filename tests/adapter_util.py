"""The adapters' and the 8-bit form's definitions in 64 bits, written plainly, and bounds on what rounding may add."""
from __future__ import annotations

import numpy as np

import synth

NP = {"f16": np.float16, "f32": np.float32}
HALF_STEP = {"f16": 2.0 ** -11, "f32": 2.0 ** -24}
SMALLEST = {"f16": 2.0 ** -25, "f32": 2.0 ** -150}      # half of the smallest step


class Problem:
    """A block-pruned layer, slots with adapters, and tokens that name them."""

    def __init__(self, dtype, m, k, n, ranks, max_rank, order="runs", relu=False, bm=16, bk=16, keep=0.6, seed=0):
        rs = np.random.RandomState(seed)
        np_dt = NP[dtype]
        self.dtype, self.m, self.k, self.n, self.max_rank, self.slots = dtype, m, k, n, max_rank, len(ranks)
        self.layer = synth.random_block_layer("adapted", m, k, n, bm, bk, dtype, keep, keep, seed=seed + 1, relu=relu)
        self.relu = relu
        self.ranks = list(ranks)                        # 0: the slot is left empty
        self.a = [(rs.standard_normal((r, k)) / np.sqrt(k)).astype(np_dt) for r in ranks]
        self.b = [(rs.standard_normal((m, r)) / np.sqrt(max(r, 1))).astype(np_dt) for r in ranks]
        self.c = [float(np.float32(s)) for s in rs.uniform(0.3, 2.0, len(ranks))]
        self.x = (rs.standard_normal((k, n)) * np.exp(rs.standard_normal((k, 1)))).astype(np_dt)
        self.dy = rs.standard_normal((m, n)).astype(np_dt)
        choices = np.arange(-1, len(ranks))
        if order == "one":
            s = np.zeros(n, np.int32)
        elif order == "none":
            s = np.full(n, -1, np.int32)
        elif order == "runs":
            s = np.sort(rs.choice(choices, n))
        elif order == "mixed":
            s = rs.choice(choices, n)
        else:                                           # values that are no slot among them
            s = rs.choice(np.concatenate([choices, [len(ranks), 2 ** 31 - 1, -2 ** 31]]), n)
        self.slot_of = s.astype(np.int32)

    def wd(self):
        return np.where(self.layer.keep_matrix(), self.layer.weights.astype(NP[self.dtype]).astype(np.float64), 0.0)

    def tokens(self, s):
        return np.flatnonzero(self.slot_of == s) if self.ranks[s] else np.zeros(0, int)

    def forward(self):
        """(y, bound on its error)."""
        x, wd = self.x.astype(np.float64), self.wd()
        bias = self.layer.bias.astype(np.float64)[:, None]
        y, size = wd @ x + bias, np.abs(wd) @ np.abs(x) + np.abs(bias)
        for s in range(self.slots):
            t = self.tokens(s)
            a, b = self.a[s].astype(np.float64), self.b[s].astype(np.float64)
            y[:, t] += self.c[s] * (b @ (a @ x[:, t]))
            size[:, t] += abs(self.c[s]) * (np.abs(b) @ (np.abs(a) @ np.abs(x[:, t])))
        if self.relu:
            y = np.maximum(y, 0.0)
        # every product and sum in binary32, in any order: k + rank terms, and what the two parts of u leave out (2^-20 of it, 16 * 2^-24)
        return y, HALF_STEP[self.dtype] * np.abs(y) + SMALLEST[self.dtype] + (2 * self.k + 2 * self.max_rank + 16) * 2.0 ** -24 * size

    def backward(self, x_held, positive, which):
        """(dx, dA, dB) and bounds, from x as it is held and the ReLU's gate (None: no ReLU)."""
        g = self.dy.astype(np.float64)
        if positive is not None:
            g = np.where(positive, g, 0.0)
        x, held, wd = self.x.astype(np.float64), x_held.astype(np.float64), self.wd()
        dx, size = wd.T @ g, np.abs(wd).T @ np.abs(g)
        da, db = np.zeros((len(which), self.max_rank, self.k)), np.zeros((len(which), self.m, self.max_rank))
        da_size, db_size = np.zeros_like(da), np.zeros_like(db)
        for s in range(self.slots):
            t = self.tokens(s)
            a, b, c = self.a[s].astype(np.float64), self.b[s].astype(np.float64), self.c[s]
            dx[:, t] += c * (a.T @ (b.T @ g[:, t]))
            size[:, t] += abs(c) * (np.abs(a).T @ (np.abs(b).T @ np.abs(g[:, t])))
        for i, s in enumerate(which):
            if not 0 <= s < self.slots:
                continue
            t, r = self.tokens(s), self.ranks[s]
            a, b, c = self.a[s].astype(np.float64), self.b[s].astype(np.float64), self.c[s]
            gt = g[:, t]
            da[i, :r] = c * ((b.T @ gt) @ held[:, t].T)
            db[i, :, :r] = c * (gt @ (a @ x[:, t]).T)
            da_size[i, :r] = abs(c) * ((np.abs(b).T @ np.abs(gt)) @ np.abs(held[:, t]).T)
            db_size[i, :, :r] = abs(c) * (np.abs(gt) @ (np.abs(a) @ np.abs(x[:, t])).T)
        terms = 2 * self.m + 2 * self.max_rank + 16
        bounds = (HALF_STEP[self.dtype] * np.abs(dx) + SMALLEST[self.dtype] + terms * 2.0 ** -24 * size,
                  (2 * self.m + 2 * self.n + 32) * 2.0 ** -24 * da_size, (2 * self.k + 2 * self.n + 32) * 2.0 ** -24 * db_size)
        return (dx, da, db), bounds


def held8(x):
    """What the 8-bit form of x [rows, n] stands for, one block at a time."""
    out = np.empty(x.shape, np.float64)
    for b in range(0, x.shape[1], 128):
        for r in range(x.shape[0]):
            v = x[r, b:b + 128].astype(np.float64)
            if not np.isfinite(v).all():
                out[r, b:b + 128] = np.nan
                continue
            e = -126
            top = np.abs(v).max()
            if top > 0:
                e = max(e, int(np.floor(np.log2(top))) - 8)
                while top > 127.0 * 2.0 ** e:
                    e += 1
            q = np.rint(v / 2.0 ** e)
            q = np.where((q == 0) & (v != 0), np.sign(v), q)
            out[r, b:b + 128] = q * 2.0 ** e
    return out


def assert_within(got, want, bound, what):
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = np.abs(got - want)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, first at {tuple(np.argwhere(bad)[0])}: {got[bad][0]} for {want[bad][0]}, bound {bound[bad][0]:.3g}"
