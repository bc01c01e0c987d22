"""Rotation of queries and keys over several axes, the norm of their heads, and attention with a sliding window and first tokens
that stay visible, against the fp64 oracle (needs a GPU).

Tolerances count roundings: u = 2^-8 relative for a value stored in bf16, 2^-24 in fp32 (half a step), and w = 2^-24 for every fp32
operation on the way, as worst cases of the sums that they enter."""
import numpy as np
import pytest

from oracle import window_oracle as wo
from paper_2605_25451_amd import binding as bm

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "fp32"]
W = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "fp32": W}


def torch_of(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(torch_of(dtype))).cuda()


def host(t):
    return t.double().cpu().numpy()


def rounded(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float64)).to(torch_of(dtype)).double().numpy()


def check(got, want, bound, what):
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), f"{what}: {off.max()} past the bound, {np.abs(got - want).max()} off"


# ---- rotation and norm ------------------------------------------------------------------------------

ROTARY = [  # tokens, q heads, kv heads, head_dim, pairs, own frequencies
    (1, 1, 1, 8, [4], False), (1, 32, 8, 128, [16, 24, 24], False), (7, 5, 1, 16, [3, 0, 5], True), (67, 16, 16, 72, [18, 18], True),
    (130, 3, 0, 64, [32], False), (129, 0, 2, 40, [7, 6, 4, 3], False), (300, 8, 2, 24, [1, 11], False), (33, 2, 2, 256, [128], False),
    (515, 6, 2, 32, [5, 5, 6], True), (1025, 12, 4, 64, [8, 12, 12], False), (2049, 2, 1, 48, [24], False)]


class Rotary:
    def __init__(self, dtype, norm, T, Hq, Hkv, dh, pairs, own, seed=0, pad=0, far=1 << 17):
        import torch
        rng = np.random.default_rng(seed)
        self.dtype, self.norm, self.shape = dtype, norm, (T, Hq, Hkv, dh)
        self.H, self.ld = Hq + Hkv, (Hq + Hkv) * dh + pad
        self.eps = 1e-5
        self.desc = bm.make_qk_rotary_desc(0 if dtype == "bf16" else 1, Hq, Hkv, dh, pairs, 10000.0, own, norm, self.eps)
        self.pos = rng.integers(-far, far, (len(pairs), T)).astype(np.int32)
        self.pos[:, ::3] %= 50
        self.far = np.abs(self.pos.astype(np.float64)).max()
        self.a = wo.angles(self.pos, pairs, 10000.0, own)
        self.x = rounded(rng.standard_normal((T, self.H, dh)) * rng.uniform(0.2, 3.0, (T, 1, 1)), dtype)
        self.dz = rounded(rng.standard_normal((T, self.H, dh)), dtype)
        self.gain = [rounded(1 + 0.3 * rng.standard_normal(dh), dtype) for _ in range(2)]
        self.dgain = rng.standard_normal((2, dh)).astype(np.float32)
        self.rows = lambda v: torch.cat([dev(v.reshape(T, -1), dtype), torch.full((T, pad), float("nan"), device="cuda", dtype=torch_of(dtype))], 1)
        self.sides = [slice(0, Hq), slice(Hq, self.H)]

    def halves(self, t):
        T, Hq, Hkv, dh = self.shape
        return t, t[:, Hq * dh:] if Hkv else t

    def gains(self):
        return [dev(g, self.dtype) for g in self.gain] if self.norm else [None, None]

    def forward(self, in_place=False):
        import torch
        x = self.rows(self.x)
        out = x if in_place else torch.full_like(x, float("nan"))
        bm.qk_rotary_forward(self.desc, self.shape[0], *self.halves(x), self.ld, dev(self.pos), *self.gains(), *self.halves(out), self.ld)
        return out

    def check_forward(self, out):
        T, Hq, Hkv, dh = self.shape
        h = dh // 2
        for g, side in zip(self.gain, self.sides):
            g = g if self.norm else None
            want = wo.rotary_forward(self.x[:, side], self.a, g, self.eps)
            y = np.abs(wo.rotary_forward(self.x[:, side], np.zeros_like(self.a), g, self.eps))
            both = np.concatenate([y[..., :h] + y[..., h:]] * 2, -1)
            # cosine and sine to 16 w, their angle to far * 2^-50; the norm's sum of up to 16 + 5 terms a lane and its root
            bound = U[self.dtype] * np.abs(want) + both * ((40 if self.norm else 16) * W + self.far * 2.0 ** -50)
            check(host(out)[:, :self.H * dh].reshape(T, self.H, dh)[:, side], want, bound, "rotated")

    def backward(self, place=None):
        import torch
        T = self.shape[0]
        x, dz = self.rows(self.x), self.rows(self.dz)
        out = {None: torch.full_like(x, float("nan")), "x": x, "dz": dz}[place]
        dg = [dev(d) for d in self.dgain]
        n = bm.qk_rotary_backward_scratch_bytes(self.desc, T)
        scratch = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
        raw = self.halves(x) if self.norm else (None, None)
        bm.qk_rotary_backward(self.desc, T, *raw, self.ld, dev(self.pos), *self.gains(), *self.halves(dz), self.ld, *self.halves(out),
                              self.ld, *(dg if self.norm else (None, None)), scratch, n)
        return out, dg

    def check_backward(self, out, dg):
        T, Hq, Hkv, dh = self.shape
        h = dh // 2
        for i, side in enumerate(self.sides):
            if side.stop == side.start:
                continue
            g = self.gain[i] if self.norm else None
            x, dz = self.x[:, side], self.dz[:, side]
            want, want_g = wo.rotary_backward(x, self.a, dz, g, self.eps)
            d = np.abs(dz)
            both = np.concatenate([d[..., :h] + d[..., h:]] * 2, -1)
            rel = 80 * W + self.far * 2.0 ** -50
            bound = U[self.dtype] * np.abs(want)
            if self.norm:
                r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + self.eps)
                n, e = np.abs(x * r), both * np.abs(g)
                bound = bound + rel * r * (e + n * (e * n).mean(-1, keepdims=True))
                # sums of at most T x heads terms, in chains of a few hundred
                bound_g = (512 * W + rel) * (both * n).sum((0, 1)) + 4 * W * np.abs(self.dgain[i])
                check(host(dg[i]), self.dgain[i].astype(np.float64) + want_g, bound_g, "gain")
            else:
                bound = bound + rel * both
            check(host(out)[:, :self.H * dh].reshape(T, self.H, dh)[:, side], want, bound, "gradient")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_rotary(case, norm, dtype):
    r = Rotary(dtype, norm, *case)
    r.check_forward(r.forward())
    r.check_backward(*r.backward())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("norm", [False, True])
def test_rotary_in_place_and_in_wider_rows(norm, dtype):
    import torch
    r = Rotary(dtype, norm, 133, 6, 2, 72, [10, 26], False, seed=1, pad=24)
    out = r.forward()
    assert torch.equal(out[:, :r.H * 72], r.forward(in_place=True)[:, :r.H * 72])
    assert torch.isnan(out[:, r.H * 72:]).all()
    d, g = r.backward()
    for place in ("x", "dz"):
        if norm or place == "dz":
            e, f = r.backward(place)
            assert torch.equal(d[:, :r.H * 72], e[:, :r.H * 72]) and all(torch.equal(a, b) for a, b in zip(g, f))
    r.check_forward(out)
    r.check_backward(d, g)


@pytest.mark.parametrize("dtype,T,Hq,Hkv", [("bf16", 9001, 12, 3), ("fp32", 4100, 10, 6), ("bf16", 3, 60000, 20000), ("fp32", 1, 1, 40000)])
@pytest.mark.parametrize("norm", [False, True])
def test_rotary_of_many_rows(dtype, T, Hq, Hkv, norm):
    """Rows that go past the caches, several trips of a workgroup; more heads than a grid has rows."""
    r = Rotary(dtype, norm, T, Hq, Hkv, 128 if T > 3 else 8, [20, 30, 14] if T > 3 else [4], False, seed=6)
    r.check_forward(r.forward())
    r.check_backward(*r.backward())


def test_rotary_at_the_farthest_positions():
    r = Rotary("fp32", False, 40, 2, 1, 32, [8, 8], False, seed=2)
    r.pos[0, :4] = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, -2 ** 31 + 1]
    r.a, r.far = wo.angles(r.pos, [8, 8], 10000.0), 2.0 ** 31
    r.check_forward(r.forward())


def test_rotary_of_a_block():
    """One axis that counts up in every sequence is what a block does."""
    import torch
    from oracle import block_oracle as bo
    r = Rotary("fp32", False, 50, 4, 2, 64, [32], False, seed=3)
    r.pos[0] = np.concatenate([np.arange(20), np.arange(30)])
    want = bo.rope_apply(r.x, bo.rope_angles(r.pos[0].astype(np.float64), 64, 10000.0))
    assert np.abs(host(r.forward()).reshape(want.shape) - want).max() < 40 * W * np.abs(r.x).max()


def test_rotary_special_values():
    """A head with an infinity or a NaN stays by itself; a head of zeros is 0, or NaN without eps."""
    import torch
    for norm in (False, True):
        r = Rotary("bf16", norm, 9, 4, 2, 16, [8], False, seed=4)
        r.x[3, 1, 5], r.x[4, 5, 0], r.x[6, 2] = np.inf, np.nan, 0.0
        z = host(r.forward()).reshape(9, 6, 16)
        bad = np.zeros((9, 6), bool)
        bad[3, 1] = bad[4, 5] = True
        assert (np.isnan(z).any(-1) | np.isinf(z).any(-1) == bad).all()
        assert (z[6, 2] == 0).all()
    r.desc.eps = 0.0
    z = host(r.forward()).reshape(9, 6, 16)
    assert np.isnan(z[6, 2]).all() and not np.isnan(z[6, 3]).any()


def test_tied_gains_take_both_gradients():
    import torch
    r = Rotary("fp32", True, 70, 3, 2, 16, [8], False, seed=5)
    _, (dq, dk) = r.backward()
    x, dz, n = r.rows(r.x), r.rows(r.dz), bm.qk_rotary_backward_scratch_bytes(r.desc, 70)
    one, scratch = torch.zeros(16, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda")
    bm.qk_rotary_backward(r.desc, 70, *r.halves(x), r.ld, dev(r.pos), *r.gains(), *r.halves(dz), r.ld, *r.halves(x), r.ld, one, one, scratch, n)
    want = (host(dq) - r.dgain[0]) + (host(dk) - r.dgain[1])
    assert np.abs(host(one) - want).max() <= 16 * W * (np.abs(want).max() + np.abs(r.dgain).max())


# ---- sliding window ------------------------------------------------------------------------------------

class Window:
    """Sequences of (queries, keys); gap: key rows between them, which hold NaN."""

    def __init__(self, dtype, Hq, Hkv, dh, seqs, window, sinks, seed=0, gap=None, pad=0, scale=1.0):
        rng = np.random.default_rng(seed)
        self.dtype, self.heads, self.window, self.sinks, self.seqs, self.pad = dtype, (Hq, Hkv, dh), window, sinks, seqs, pad
        self.code = 0 if dtype == "bf16" else 1
        self.cu = np.concatenate([[0], np.cumsum([a for a, _ in seqs])]).astype(np.int32)
        own = gap is not None or any(a != b for a, b in seqs)
        lens, gap = [b for _, b in seqs], gap or 0
        self.begin = np.array([sum(lens[:i]) + gap * (i + 1) for i in range(len(lens))], np.int32)
        self.end = (self.begin + lens).astype(np.int32)
        self.own = own
        self.Tq, self.Tk = int(self.cu[-1]), int(self.end[-1]) + gap
        if not own:
            self.Tk = self.Tq
        draw = lambda n, h, s=1.0: rounded(rng.standard_normal((n, h, dh)) * s, dtype)
        self.q, self.d_o = draw(self.Tq, Hq, scale), draw(self.Tq, Hq)
        self.k, self.v = draw(self.Tk, Hkv, scale), draw(self.Tk, Hkv)
        self.inside = np.zeros(self.Tk, bool)
        for b, e in zip(self.begin, self.end):
            self.inside[b:e] = True

    def rows(self, x, holes=False):
        import torch
        t = dev(x.reshape(len(x), -1), self.dtype)
        if holes:
            t[dev(~self.inside)] = float("nan")
        return torch.cat([t, torch.full((len(x), self.pad), float("nan"), device="cuda", dtype=t.dtype)], 1)

    def common(self):
        Hq, Hkv, dh = self.heads
        self.keep = [self.rows(self.q), self.rows(self.k, True), self.rows(self.v, True), dev(self.cu)] + \
            ([dev(self.begin), dev(self.end)] if self.own else [None, None])
        q, k, v, cu, b, e = self.keep
        head = (self.code, self.window, self.sinks, Hq, Hkv, dh, q, Hq * dh + self.pad, k, v, Hkv * dh + self.pad)
        return head, (cu, self.cu, b, e, self.begin if self.own else None, self.end if self.own else None, len(self.seqs))

    def sizes(self):
        return (self.code, self.window, self.sinks, *self.heads, len(self.seqs), self.Tq, int(self.end.max()) if self.own else self.Tk)

    def scratch(self, n):
        import torch
        return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")

    def forward(self):
        """o and lse with a row and a column more than they need"""
        import torch
        Hq, _, dh = self.heads
        self.o = torch.full((self.Tq + 1, Hq * dh), float("nan"), device="cuda", dtype=torch_of(self.dtype))
        self.lse = torch.full((Hq * self.Tq + 5,), float("nan"), device="cuda")
        head, offsets = self.common()
        n = bm.window_attention_scratch_bytes(*self.sizes())
        self.fwd_work = self.scratch(n)
        self.fwd = lambda: bm.window_attention_forward(*head, *offsets, self.o, self.lse, self.fwd_work, n)
        self.fwd()
        return self.o, self.lse

    def backward(self):
        import torch
        Hq, Hkv, dh = self.heads
        o, lse = self.oracle_forward()
        self.o_in, self.lse_in = dev(np.concatenate(o).reshape(self.Tq, -1), self.dtype), dev(np.concatenate(lse, 1).astype(np.float32))
        self.d_in = dev(self.d_o.reshape(self.Tq, -1), self.dtype)
        wide = lambda n, H: torch.full((n, H * dh + self.pad), 7.0, device="cuda", dtype=torch_of(self.dtype))
        self.grads = wide(self.Tq + 1, Hq), wide(self.Tk, Hkv), wide(self.Tk, Hkv)
        head, offsets = self.common()
        n = bm.window_attention_backward_scratch_bytes(*self.sizes())
        self.bwd_work = self.scratch(n)
        self.bwd = lambda: bm.window_attention_backward(*head, self.o_in, self.d_in, self.lse_in, *offsets, self.grads[0], Hq * dh + self.pad,
                                                        self.grads[1], self.grads[2], Hkv * dh + self.pad, self.bwd_work, n)
        self.bwd()
        return self.grads

    def each(self):
        for s, (lq, lk) in enumerate(self.seqs):
            yield slice(int(self.cu[s]), int(self.cu[s + 1])), slice(int(self.begin[s]) if self.own else int(self.cu[s]),
                                                                     int(self.end[s]) if self.own else int(self.cu[s + 1]))

    def oracle_forward(self):
        got = [wo.attention(self.q[a], self.k[b], self.v[b], self.window, self.sinks) for a, b in self.each()]
        return [o for o, _ in got], [l for _, l in got]

    def check_forward(self, o, lse):
        Hq, Hkv, dh = self.heads
        u, group = U[self.dtype], Hq // Hkv
        o, lse = host(o), host(lse)
        assert np.isnan(o[self.Tq:]).all() and np.isnan(lse[Hq * self.Tq:]).all(), "rows behind the last one"
        o, lse = o[:self.Tq].reshape(self.Tq, Hq, dh), lse[:Hq * self.Tq].reshape(Hq, self.Tq)
        for (a, b), want_o, want_l in zip(self.each(), *self.oracle_forward()):
            for h in range(Hq):
                q, k, v = self.q[a, h], self.k[b, h // group], self.v[b, h // group]
                if not len(q):
                    continue
                p, _ = wo.probabilities(q, k, self.window, self.sinks)
                s = (np.abs(q) @ np.abs(k).T).max() * dh ** -0.5        # a score's error: dh products and sums, and 4 in base 2
                rel = (dh + 4) * W * s
                check(lse[h, a], want_l[h], 1.05 * (rel + (len(k) + 8) * W + 8 * W * np.abs(want_l[h])), "lse")
                # a probability: rounded to u on the matrix cores, its score's error, the sum of them
                bound = (u + 2 * rel + (2 * len(k) + 16) * W) * (p @ np.abs(v)) + u * np.abs(want_o[:, h])
                check(o[a, h], want_o[:, h], 1.05 * bound, "o")

    def check_backward(self, dq, dk, dv):
        Hq, Hkv, dh = self.heads
        u, group, scale = U[self.dtype], Hq // Hkv, dh ** -0.5
        assert (host(dq)[self.Tq:] == 7).all(), "a row behind the last one"
        for x in (dk, dv):
            assert (host(x)[~self.inside if self.own else slice(0, 0)] == 7).all(), "rows between the sequences"
        for x, H in ((dq, Hq), (dk, Hkv), (dv, Hkv)):
            assert (host(x)[:, H * dh:] == 7).all(), "columns beside the rows"
        dq, dk, dv = (host(x)[:n, :H * dh].reshape(n, H, dh) for x, n, H in ((dq, self.Tq, Hq), (dk, self.Tk, Hkv), (dv, self.Tk, Hkv)))
        for a, b in self.each():
            q, k, v, d_o = self.q[a], self.k[b], self.v[b], self.d_o[a]
            wq, wk, wv = wo.attention_backward(q, k, v, d_o, self.window, self.sinks)
            eq, ek, ev = u * np.abs(wq), u * np.abs(wk), u * np.abs(wv)
            n = len(k) + len(q) * group
            for h in range(Hq if len(q) else 0):
                c = h // group
                p, _ = wo.probabilities(q[:, h], k[:, c], self.window, self.sinks)
                dp = d_o[:, h] @ v[:, c].T
                delta = (p * dp).sum(1, keepdims=True)
                o = p @ v[:, c]
                s = (np.abs(q[:, h]) @ np.abs(k[:, c]).T).max() * scale
                rel = 2 * u + 2 * ((dh + 4) * W * s + 8 * W + 2.0 ** -23 * 16)     # of a probability and of dS, which bf16 rounds as well
                # dP - delta: dh products and sums each; o as it was stored
                base = p * ((dh + 2) * W * (np.abs(d_o[:, h]) @ np.abs(v[:, c]).T) + (u + (dh + 2) * W) * (np.abs(o) * np.abs(d_o[:, h])).sum(1, keepdims=True))
                err = (rel + n * W) * np.abs(p * (dp - delta)) + base
                eq[:, h] += scale * err @ np.abs(k[:, c])
                ek[:, c] += scale * err.T @ np.abs(q[:, h])
                ev[:, c] += (rel + n * W) * (p.T @ np.abs(d_o[:, h]))
            check(dq[a], wq, 1.05 * eq + 1e-30, "dq")
            check(dk[b], wk, 1.05 * ek + 1e-30, "dk")
            check(dv[b], wv, 1.05 * ev + 1e-30, "dv")


pack = lambda *lens: [(n, n) for n in lens]
WINDOWS = [  # q heads, kv heads, sequences, window, sinks
    (1, 1, pack(1), 1, 0), (4, 4, pack(2, 1, 3), 2, 1), (4, 2, pack(130, 64, 257), 64, 0), (4, 1, pack(130, 65, 257), 63, 5),
    (2, 2, pack(300), 1, 0), (2, 2, pack(300), 1, 128), (4, 2, pack(200, 129), 1 << 30, 3), (3, 3, pack(511, 127), 129, 64),
    (8, 2, pack(1100), 70, 4), (2, 1, pack(640, 1, 700), 128, 127), (2, 2, pack(513), 400, 1)]
SUFFIXES = [
    (8, 2, [(1, 1)], 5, 2), (8, 2, [(1, 1000), (1, 3), (1, 64)], 100, 4), (4, 4, [(5, 5), (0, 7), (0, 0), (130, 400)], 90, 33),
    (4, 1, [(3, 900), (2, 129), (70, 71)], 300, 0), (2, 2, [(600, 900), (1, 200)], 64, 9), (8, 1, [(1, 4000), (4, 2100)], 3000, 128)]
HEADS = [("bf16", 64), ("bf16", 72), ("bf16", 128), ("bf16", 32), ("fp32", 64), ("fp32", 72), ("fp32", 16)]


@pytest.mark.parametrize("dtype,dh", HEADS)
@pytest.mark.parametrize("case", WINDOWS, ids=lambda c: "%d-%d-%s-%d-%d" % (c[0], c[1], "+".join(str(a) for a, _ in c[2]), *c[3:]))
def test_window_of_a_pack(case, dtype, dh):
    Hq, Hkv, seqs, window, sinks = case
    x = Window(dtype, Hq, Hkv, dh, seqs, window, sinks)
    x.check_forward(*x.forward())
    x.check_backward(*x.backward())


@pytest.mark.parametrize("dtype,dh", HEADS)
@pytest.mark.parametrize("case", SUFFIXES, ids=lambda c: "%d-%d-%s-%d-%d" % (c[0], c[1], "+".join("%d.%d" % s for s in c[2]), *c[3:]))
def test_window_of_the_last_queries(case, dtype, dh):
    Hq, Hkv, seqs, window, sinks = case
    x = Window(dtype, Hq, Hkv, dh, seqs, window, sinks, seed=1, gap=3)
    x.check_forward(*x.forward())
    x.check_backward(*x.backward())


TOKENS = [
    (32, 1, [(1, 5000)], 4500, 100), (16, 2, [(4, 700), (1, 1), (3, 3), (2, 1500)], 1000, 33), (12, 12, [(1, 2300), (1, 40)], 2000, 1),
    (6, 2, [(1, 100 + 31 * i) for i in range(70)], 1200, 5), (2, 1, [(1 + i % 16, 20 + i * i % 900) for i in range(66)], 64, 65),
    (2, 2, [(i % 2, 1 + i * 37 % 700) for i in range(600)], 600, 2)]


@pytest.mark.parametrize("dtype,dh", HEADS + [("bf16", 8), ("fp32", 128), ("fp32", 8), ("fp32", 32)])
@pytest.mark.parametrize("case", TOKENS, ids=lambda c: "%d-%d-%d-%d-%d" % (c[0], c[1], len(c[2]), *c[3:]))
def test_window_of_few_queries(case, dtype, dh):
    """Keys split over workgroups, with and without the table of the sequences' parts in the kernel's arguments."""
    Hq, Hkv, seqs, window, sinks = case
    x = Window(dtype, Hq, Hkv, dh, seqs, window, sinks, seed=9, gap=2)
    x.check_forward(*x.forward())


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 72), ("bf16", 128), ("fp32", 32)])
def test_window_in_wider_rows(dtype, dh):
    x = Window(dtype, 4, 2, dh, pack(100, 333), 50, 2, seed=2, pad=8)
    x.check_forward(*x.forward())
    x.check_backward(*x.backward())


@pytest.mark.parametrize("dtype,dh,sinks", [("bf16", 64, 2), ("bf16", 128, 0), ("bf16", 128, 6), ("fp32", 16, 2)])
def test_window_of_many_sequences(dtype, dh, sinks):
    """More sequences than a table in the kernel's arguments holds, a long one among them."""
    lens = [1 + (i * 7) % 13 for i in range(80)]
    lens[40] = 1300
    x = Window(dtype, 2, 1, dh, pack(*lens), 37, sinks, seed=3)
    x.check_forward(*x.forward())
    x.check_backward(*x.backward())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64)])
@pytest.mark.parametrize("sinks", [0, 5, 90])
@pytest.mark.parametrize("heads,seqs,window", [((16, 16), [(2100, 2100)], 530), ((16, 8), [(2200, 2300)], 530),
                                               ((12, 6), [(1500, 1500), (40, 900), (700, 1111)], 300),
                                               ((12, 6), [(1500, 1500), (40, 900), (700, 1111)], 60)], ids=str)
def test_window_of_long_sequences(heads, seqs, window, sinks, dtype, dh):
    """Packs that fill the chip: 256 keys to a workgroup of dK/dV at head size 128, dQ of a narrow window in a launch of its own, q heads of a group in
    parts, first keys in parts of 512 rows."""
    x = Window(dtype, *heads, dh, seqs, window, sinks, seed=14, gap=2 if seqs[0][0] != seqs[0][1] else None)
    x.check_forward(*x.forward())
    x.check_backward(*x.backward())


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 72), ("bf16", 128), ("fp32", 64)])
def test_a_wide_window_is_causal_attention(dtype, dh):
    """Strong scores as well: the largest in a row decides."""
    import torch
    seqs, Hq, Hkv = pack(257, 90), 4, 2
    x = Window(dtype, Hq, Hkv, dh, seqs, 300, 0, seed=4, scale=3.0)
    o, lse = x.forward()
    x.check_forward(o, lse)
    rows = torch.cat([x.rows(x.q), x.rows(x.k), x.rows(x.v)], 1)
    o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
    bm.attention_forward(x.code, 1, Hq, Hkv, dh, rows, rows[:, Hq * dh:], rows[:, (Hq + Hkv) * dh:], (Hq + 2 * Hkv) * dh, dev(x.cu), x.cu,
                         2, x.Tq, 257, o2, lse2)
    # Both are within the bound of the definition, so no further than two bounds apart.  (In fp32 they add a score's products in different
    # orders: at |q| |k| / sqrt(dh) = 15 each sum is off by up to (dh + 4) W 15 = 6e-5, and a probability by as much of itself, which is 1000
    # of its own roundings: equality to a few roundings would ask for the same order.)
    x.check_forward(o2, lse2)


@pytest.mark.parametrize("seqs", [[(2, 1400), (1, 900), (1, 70)], [(40, 1400), (300, 900)], [(1, 60 + 11 * i) for i in range(70)]], ids=["few", "many", "long list"])
@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 72), ("bf16", 128), ("fp32", 32), ("fp32", 128)])
@pytest.mark.parametrize("window,sinks", [(40, 3), (37, 0), (65, 70)])
def test_keys_that_no_query_sees_are_not_read(window, sinks, dtype, dh, seqs):
    """Infinities and NaN in them, as an emptied part of a cache holds them."""
    import torch
    x = Window(dtype, 4, 2, dh, seqs, window, sinks, seed=5, gap=9)
    o, lse = (t.clone() for t in x.forward())
    for (n, _), b, e in zip(seqs, x.begin, x.end):
        x.keep[1][b + sinks:max(b + sinks, e - n - window + 1)] = float("nan")
        x.keep[2][b + sinks:max(b + sinks, e - n - window + 1)] = float("inf")
    x.fwd()
    assert torch.equal(o[:x.Tq], x.o[:x.Tq]) and torch.equal(lse[:4 * x.Tq], x.lse[:4 * x.Tq])


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("fp32", 32)])
@pytest.mark.parametrize("queries", [(1, 2), (1, 90)])
def test_sequences_that_share_keys_in_any_order(dtype, dh, queries):
    """A common beginning, as several answers to one question have it, and a slot in front of the others."""
    x = Window(dtype, 8, 2, dh, [(queries[0], 300), (queries[1], 320), (1, 100)], 80, 5, seed=10, gap=3)
    x.begin[1], x.end[1] = x.begin[0], x.begin[0] + 320
    x.begin[0], x.end[0], x.begin[2], x.end[2] = x.begin[2], x.end[2], x.begin[0], x.end[0]
    x.seqs = [(q, int(e - b)) for (q, _), b, e in zip(x.seqs, x.begin, x.end)]
    x.inside[:] = False
    for b, e in zip(x.begin, x.end):
        x.inside[b:e] = True
    x.check_forward(*x.forward())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 72), ("fp32", 64)])
@pytest.mark.parametrize("queries", [(1, 1), (2, 130)])
def test_keys_far_into_a_cache(dtype, dh, queries):
    """Rows whose offsets pass 2^32 bytes; the rest of the cache holds NaN."""
    import torch
    Hq, Hkv, lens, window, sinks, ld = 8, 2, (700, 333), 150, 3, 1024
    rows = (1 << 33) // (ld * (2 if dtype == "bf16" else 4)) // 2
    near = Window(dtype, Hq, Hkv, dh, list(zip(queries, lens)), window, sinks, seed=11, gap=1)
    o, lse = near.forward()
    near.check_forward(o, lse)
    begin = np.array([rows - 1100, rows - 350], np.int32)
    end = (begin + lens).astype(np.int32)
    big = [torch.full((rows, ld), float("nan"), device="cuda", dtype=torch_of(dtype)) for _ in range(2)]
    for b, nb, n in zip(begin, near.begin, lens):
        for t, src in zip(big, (near.k, near.v)):
            t[b:b + n, :Hkv * dh] = dev(src[nb:nb + n].reshape(n, -1), dtype)
    n = bm.window_attention_scratch_bytes(near.code, window, sinks, Hq, Hkv, dh, 2, near.Tq, int(end[1]))
    o2, lse2 = torch.empty_like(o[:near.Tq]), torch.empty(Hq * near.Tq, device="cuda")
    bm.window_attention_forward(near.code, window, sinks, Hq, Hkv, dh, near.rows(near.q), Hq * dh, big[0], big[1], ld, dev(near.cu), near.cu, dev(begin),
                                dev(end), begin, end, 2, o2, lse2, near.scratch(n), n)
    assert torch.equal(o2, o[:near.Tq]) and torch.equal(lse2, lse[:Hq * near.Tq])


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_window_replays_from_a_graph_and_repeats(dtype, dh):
    """The same bits again, from a graph with eager work between the replays, and on another stream."""
    import torch
    x = Window(dtype, 4, 2, dh, pack(700, 130), 60, 4, seed=6)
    x.forward()
    x.backward()
    want = [t.clone() for t in (x.o, x.lse, *x.grads)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        x.fwd()
        x.bwd()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t in (x.o, x.lse, *x.grads):
            t[:x.Tq] = 7.0 if t.dim() == 2 else float("nan")
        x.fwd_work.fill_(255)
        x.bwd_work.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((x.o, x.lse, *x.grads), want):
            assert torch.equal(got[:x.Tq], ref[:x.Tq])


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("fp32", 64)])
@pytest.mark.parametrize("S", [3, 70])
def test_tokens_replay_from_graphs_that_run_at_the_same_time(S, dtype, dh):
    """Two graphs with workspaces of their own, replayed side by side, lists that grow by nothing; then once more in eager mode."""
    import torch
    xs = [Window(dtype, 8, 2, dh, [(1 + i % 2, 40 + (i * 211 + 97 * j) % 1900) for i in range(S)], 900, 5, seed=12 + j, gap=1) for j in range(2)]
    want = [tuple(t.clone() for t in x.forward()) for x in xs]
    for x in xs:
        x.check_forward(x.o, x.lse)
    streams, graphs = [torch.cuda.Stream() for _ in xs], [torch.cuda.CUDAGraph() for _ in xs]
    for x, st, g in zip(xs, streams, graphs):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=st):
            x.fwd()
    for _ in range(3):
        for x in xs:
            x.o[:x.Tq], x.lse[:8 * x.Tq] = 7.0, 7.0
            x.fwd_work.fill_(255)
        torch.cuda.synchronize()
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for x, (o, lse) in zip(xs, want):
            assert torch.equal(x.o[:x.Tq], o[:x.Tq]) and torch.equal(x.lse[:8 * x.Tq], lse[:8 * x.Tq])
    xs[0].fwd()
    assert torch.equal(xs[0].o[:xs[0].Tq], want[0][0][:xs[0].Tq])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("norm", [False, True])
def test_rotary_replays_from_a_graph(norm, dtype):
    import torch
    r = Rotary(dtype, norm, 700, 6, 2, 64, [8, 12, 12], False, seed=13)
    x, dz, pos, gains = r.rows(r.x), r.rows(r.dz), dev(r.pos), r.gains()
    z, dx, dg = torch.zeros_like(x), torch.zeros_like(x), [torch.zeros(64, device="cuda") for _ in range(2)]
    n = bm.qk_rotary_backward_scratch_bytes(r.desc, 700)
    work = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    raw = r.halves(x) if norm else (None, None)

    def both():
        bm.qk_rotary_forward(r.desc, 700, *r.halves(x), r.ld, pos, *gains, *r.halves(z), r.ld)
        bm.qk_rotary_backward(r.desc, 700, *raw, r.ld, pos, *gains, *r.halves(dz), r.ld, *r.halves(dx), r.ld, *(dg if norm else (None, None)), work, n)
    both()
    want = [t.clone() for t in (z, dx, *dg)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        both()
    for _ in range(3):
        for t in (z, dx, *dg):
            t.zero_()
        work.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((z, dx, *dg), want))


# ---- one after another, as a model uses them -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_rotation_and_window_together(dtype):
    """Projected rows -> norm and rotation -> windowed attention, and back."""
    import torch
    Hq, Hkv, dh, seqs, window, sinks = 4, 2, 64, pack(190, 77), 48, 2
    T = 267
    r = Rotary(dtype, True, T, Hq, Hkv, dh, [8, 12, 12], False, seed=7, far=300)
    w = Window(dtype, Hq, Hkv, dh, seqs, window, sinks, seed=8)
    ld, both, t = (Hq + 2 * Hkv) * dh, (Hq + Hkv) * dh, torch_of(dtype)
    raw = torch.cat([r.rows(r.x), w.rows(w.v)], 1)
    turned = raw.clone()
    pos, gains, cu = dev(r.pos), r.gains(), dev(w.cu)
    parts = lambda x: (x, x[:, Hq * dh:], x[:, both:])
    bm.qk_rotary_forward(r.desc, T, raw, raw[:, Hq * dh:], ld, pos, *gains, turned, turned[:, Hq * dh:], ld)
    o, lse = torch.empty((T, Hq * dh), device="cuda", dtype=t), torch.empty((Hq, T), device="cuda")
    q, k, v = parts(turned)
    common = (w.code, window, sinks, Hq, Hkv, dh, q, ld, k, v, ld)
    n = bm.window_attention_scratch_bytes(w.code, window, sinks, Hq, Hkv, dh, 2, T, T)
    bm.window_attention_forward(*common, cu, w.cu, None, None, None, None, 2, o, lse, w.scratch(n), n)
    grads = torch.empty_like(raw)
    n = bm.window_attention_backward_scratch_bytes(w.code, window, sinks, Hq, Hkv, dh, 2, T, T)
    d_o = dev(w.d_o.reshape(T, -1), dtype)
    bm.window_attention_backward(*common, o, d_o, lse, cu, w.cu, None, None, None, None, 2, grads, ld, *parts(grads)[1:], ld, w.scratch(n), n)
    dg = [torch.zeros(dh, device="cuda") for _ in range(2)]
    n = bm.qk_rotary_backward_scratch_bytes(r.desc, T)
    bm.qk_rotary_backward(r.desc, T, raw, raw[:, Hq * dh:], ld, pos, *gains, grads, grads[:, Hq * dh:], ld, grads, grads[:, Hq * dh:], ld, *dg,
                          w.scratch(n), n)
    # the oracle's chain, without a rounding between
    z = [wo.rotary_forward(r.x[:, s], r.a, g, r.eps) for s, g in zip(r.sides, r.gain)]
    want_o, back = [], []
    for a, _ in w.each():
        want_o.append(wo.attention(z[0][a], z[1][a], w.v[a], window, sinks)[0])
        back.append(wo.attention_backward(z[0][a], z[1][a], w.v[a], w.d_o[a], window, sinks))
    dz = [np.concatenate(x) for x in zip(*back)]
    want, want_g = zip(*(wo.rotary_backward(r.x[:, s], r.a, d, g, r.eps) for s, d, g in zip(r.sides, dz, r.gain)))
    # values pass through at most four stored tensors, each off by u of its largest; sums over n keys average roundings
    tol = {"bf16": 2e-2, "fp32": 1e-5}[dtype]                # the tolerances of a block's path
    for got, ref, what in ((o, np.concatenate(want_o), "o"), (grads, np.concatenate([*want, dz[2]], 1), "dx"), (dg[0], want_g[0], "dq_gain"),
                           (dg[1], want_g[1], "dk_gain")):
        off = np.abs(host(got).reshape(ref.shape) - ref).max() / np.abs(ref).max()
        assert off <= tol, f"{what}: {off}"
