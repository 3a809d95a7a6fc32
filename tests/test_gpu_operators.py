"""The sequence operators (dropout without a stored mask, the gated linear
recurrence and its gradient, the scores' penalties, biases and masks) against
plain implementations in 64 bits, through the public entry points.

Tolerances.  eps = 2^-24 bounds the relative error of one float32 operation,
U[dtype] that of the one rounding to the storage format (half a unit in the
last place; TINY: half the spacing of its subnormals).  Each test adds up the
operations that its values go through; none is fitted to a result.
"""
import ctypes
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def pg():
    import paper_1404_1521_amd as pg
    return pg


@pytest.fixture(scope="module")
def ctx(pg):
    c = pg.Context(1000, 16, 5, 8, max_batch=1)
    c.reserve_recurrence(20_000, 2048)
    c.reserve_logits(64, 1_000_003)
    yield c
    assert c.status() == pg.OK
    c.close()


def host(t):
    return t.detach().double().cpu().numpy()


def dev(a, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]).cuda()


def strided(t, pad, shift):
    """t's values in rows t.shape[1] + pad apart that start `shift` elements in."""
    n, w = t.shape
    buf = torch.full((n * (w + pad) + shift + 8,), 77.0, dtype=t.dtype, device="cuda")
    view = buf[shift:shift + n * (w + pad)].view(n, w + pad)[:, :w]
    view.copy_(t)
    return view


def near(got, ref, bound, what=""):
    bad = ~(np.abs(got - ref) <= bound) & ~((got == ref) | (np.isnan(got) & np.isnan(ref)))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4],
                           ref[bad][:4], np.broadcast_to(bound, ref.shape)[bad][:4])


# ------------------------------------------------------------------ dropout


def philox(c, k):
    """Philox 4x32-10 of counter words c (uint64 arrays below 2^32) and key words k."""
    c = [np.asarray(x, np.uint64) for x in c]
    m = np.uint64(0xFFFFFFFF)
    k0, k1 = k
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def test_philox_reference_vectors():
    """The generator's published known answers (Random123's kat_vectors: zeros, ones)."""
    z = philox([0, 0, 0, 0], (0, 0))
    assert [int(x) for x in z] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    o = philox([0xFFFFFFFF] * 4, (0xFFFFFFFF, 0xFFFFFFFF))
    assert [int(x) for x in o] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def kept(rows, d, p, seed, site=0, first_row=0, whole=False):
    n8 = 1 if whole else -(-d // 8)
    r = np.uint64(first_row) + np.arange(rows, dtype=np.uint64)[:, None]
    g = np.full((1, 1), 0xFFFFFFFF, np.uint64) if whole else np.arange(n8, dtype=np.uint64)[None]
    r, g = np.broadcast_arrays(r, g)
    m = np.uint64(0xFFFFFFFF)
    w = philox([g, r & m, r >> np.uint64(32), np.full(r.shape, site, np.uint64)],
               (seed & 0xFFFFFFFF, seed >> 32))
    out = np.empty((rows, n8, 8), bool)
    limit = int(np.float32(p) * 65536.0 + 0.5)
    for j in range(8):
        out[:, :, j] = (w[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) >= limit
    return np.repeat(out[:, 0, :1], d, 1) if whole else out.reshape(rows, -1)[:, :d]


def dropout_ref(x, keep, p, add=None):
    limit = int(np.float32(p) * 65536.0 + 0.5)
    scale = 65536.0 / (65536 - limit) if limit < 65536 else 0.0
    y = np.where(keep, np.where(keep, x, 0) * scale, 0.0)
    size = np.abs(y) + (0 if add is None else np.abs(add))
    return (y if add is None else y + add), size


def check_dropout(got, x, keep, p, dtype, add=None):
    ref, size = dropout_ref(x, keep, p, add)
    # the scale's rounding, the product, the sum; then the format's
    near(host(got), ref, 3.01 * EPS * size + U[dtype] * (np.abs(ref) + 4 * EPS * size)
         + TINY[dtype], dtype)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (257, 8), (65, 63), (130, 64), (19, 199),
                                    (5, 256), (33, 513), (2, 4100), (1030, 24)])
def test_dropout_forms(ctx, dtype, rows, d):
    rng = np.random.default_rng([rows, d])
    x, add = dev(rng.normal(size=(rows, d)), dtype), dev(rng.normal(size=(rows, d)), dtype)
    seed = int(rng.integers(0, 1 << 62))
    for p, whole in ((0.1, False), (0.5, False), (0.3, True)):
        keep = kept(rows, d, p, seed, 3, 0, whole)
        y = ctx.dropout(x, p, seed, site=3, whole_rows=whole)
        check_dropout(y, host(x), keep, p, dtype)
        y = ctx.dropout(x, p, seed, site=3, whole_rows=whole, add=add)
        check_dropout(y, host(x), keep, p, dtype, host(add))
        g = ctx.dropout_backward(add, p, seed, site=3, whole_rows=whole)
        check_dropout(g, host(add), keep, p, dtype)
    # rows apart, starts that no vector is aligned to
    xs, adds = strided(x, 5, 3), strided(add, 2, 1)
    out = strided(torch.zeros_like(x), 3, 5)
    guard = out._base.clone()
    keep = kept(rows, d, 0.25, seed)
    ctx.dropout(xs, 0.25, seed, add=adds, out=out)
    check_dropout(out, host(x), keep, 0.25, dtype, host(add))
    out.zero_()
    assert torch.equal(out._base, guard)  # nothing outside of the rows was written
    # in place, on x and on add
    z = x.clone()
    assert ctx.dropout(z, 0.25, seed, out=z) is z
    check_dropout(z, host(x), keep, 0.25, dtype)
    z = add.clone()
    ctx.dropout(x, 0.25, seed, add=z, out=z)
    check_dropout(z, host(x), keep, 0.25, dtype, host(add))


@pytest.mark.parametrize("dtype,rows,d", [("f32", 1100, 9001), ("bf16", 1_100_000, 5),
                                          ("f16", 70_001, 123)])
def test_dropout_of_many_elements(ctx, dtype, rows, d):
    """Several groups of columns to a thread; rows of more and of fewer groups than a
    workgroup takes."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, d, device="cuda", generator=gen).to(DT[dtype])
    keep = torch.from_numpy(kept(rows, d, 0.3, 21)).cuda()
    y = ctx.dropout(x, 0.3, 21, add=x)
    limit = int(np.float32(0.3) * 65536.0 + 0.5)
    ref = torch.where(keep, x.double() * (65536 / (65536 - limit)), 0.0) + x.double()
    size = 2.5 * x.double().abs()
    bound = 3.01 * EPS * size + U[dtype] * (ref.abs() + 4 * EPS * size) + TINY[dtype]
    assert ((y.double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("d", [1, 64, 100, 128, 131])
def test_dropout_of_table_rows(pg, ctx, dtype, idt, d):
    rng = np.random.default_rng(d)
    V, rows = 301, 777
    table = dev(rng.normal(size=(V, d)), dtype)
    ids = torch.from_numpy(rng.integers(0, V, rows)).to(idt).cuda()
    x = host(table)[ids.cpu().numpy()]
    for p, whole in ((0.2, False), (0.6, True), (0.0, False)):
        keep = kept(rows, d, p, 99, 1, 0, whole)
        check_dropout(ctx.dropout(table, p, 99, site=1, ids=ids, whole_rows=whole), x, keep, p,
                      dtype)
    assert ctx.status() == pg.OK
    bad = ids.clone()
    bad[5], bad[700] = V, -1
    y = host(ctx.dropout(table, 0.2, 99, site=1, ids=bad))
    assert ctx.status() == pg.EID and ctx.status() == pg.OK
    hit = np.isnan(y).all(1)
    assert hit[[5, 700]].all() and hit.sum() == 2 and not np.isnan(y[~hit]).any()


@pytest.mark.parametrize("dtype", list(DT))
def test_dropout_limits(ctx, dtype):
    x = dev(np.random.default_rng(1).normal(size=(40, 72)), dtype)
    assert torch.equal(ctx.dropout(x, 0.0, 5), x)
    assert torch.equal(ctx.dropout(x, 1.0, 5), torch.zeros_like(x))
    assert torch.equal(ctx.dropout(x, 1.0, 5, add=x), x)
    # a probability below the 16 bits' resolution drops nothing
    assert torch.equal(ctx.dropout(x, 2.0 ** -18, 5), x)
    # what is dropped is exactly zero, also where x is not a number
    keep = torch.from_numpy(kept(40, 72, 0.5, 5)).cuda()
    for v in (math.nan, math.inf, -math.inf):
        y = ctx.dropout(torch.full_like(x, v), 0.5, 5)
        assert (y[~keep] == 0).all() and not torch.isfinite(y[keep]).any()
    e = ctx.dropout(x[:0], 0.5, 5)
    assert e.shape == (0, 72)


def test_dropout_mask_is_a_function_of_the_position(ctx):
    x = torch.ones(300, 40, device="cuda")
    whole = ctx.dropout(x, 0.4, 11, site=2)
    parts = [ctx.dropout(x[a:b], 0.4, 11, site=2, first_row=a) for a, b in
             ((0, 1), (1, 130), (130, 300))]
    assert torch.equal(whole, torch.cat(parts))
    assert torch.equal(whole.half(), ctx.dropout(x.half(), 0.4, 11, site=2))
    assert torch.equal(whole[:, :33], ctx.dropout(x[:, :33], 0.4, 11, site=2))
    far = (1 << 40) + 12345
    y = ctx.dropout(x, 0.4, (1 << 63) + 5, site=(1 << 32) - 1, first_row=far)
    check_dropout(y, host(x), kept(300, 40, 0.4, (1 << 63) + 5, (1 << 32) - 1, far), 0.4, "f32")
    assert not torch.equal(whole, ctx.dropout(x, 0.4, 11, site=3))
    assert not torch.equal(whole, ctx.dropout(x, 0.4, 12, site=2))


def test_dropout_rate(ctx):
    n = 4_000_000
    y = ctx.dropout(torch.ones(1000, n // 1000, device="cuda"), 0.1, 77)
    share = float((y == 0).double().mean())
    p = 6554 / 65536
    assert abs(share - p) < 5 * math.sqrt(p * (1 - p) / n)


def test_dropout_rows_past_32_bits(ctx):
    ld = (1 << 32) + 4096
    buf = torch.empty(ld + 256, dtype=torch.float16, device="cuda")
    x = buf.as_strided((2, 200), (ld, 1))
    x.copy_(torch.randn(2, 200, device="cuda"))
    table = buf.as_strided((2, 200), (ld, 1))
    ids = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    a = host(x)
    check_dropout(ctx.dropout(x, 0.3, 1), a, kept(2, 200, 0.3, 1), 0.3, "f16")
    check_dropout(ctx.dropout(table, 0.3, 1, ids=ids), a[[1, 0, 1]], kept(3, 200, 0.3, 1), 0.3,
                  "f16")
    ctx.dropout(x.clone(), 0.3, 1, out=x)
    check_dropout(x, a, kept(2, 200, 0.3, 1), 0.3, "f16")


def test_dropout_of_more_groups_than_a_launch_has(ctx):
    # a launch takes 2^31 groups of up to eight columns; rows on both sides of the cut,
    # and the last ones, against calls of their own rows
    rows = 2**31 + 5
    x = torch.ones(rows, 1, device="cuda", dtype=torch.bfloat16)
    ctx.dropout(x, 0.5, 71, site=3, out=x)
    torch.cuda.synchronize()
    for at in (0, 2**31 - 300, 2**31 - 3, rows - 300):
        n = min(600, rows - at)
        want = ctx.dropout(torch.ones(n, 1, device="cuda", dtype=torch.bfloat16), 0.5, 71, site=3,
                           first_row=at)
        assert torch.equal(x[at:at + n], want), at
        assert n < 300 or 0 < int((want == 0).sum()) < n
    assert ctx.status() == 0


def test_dropout_in_a_graph(pg):
    """The mask of a replay follows the device word that the program advances."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = pg.Context(1000, 16, 5, 8, max_batch=1, stream=s)
        x = torch.randn(64, 96, device="cuda")
        y, site = torch.empty_like(x), torch.zeros(1, dtype=torch.int32, device="cuda")
        c.dropout(x, 0.3, 9, site=10, site_dev=site, out=y)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.dropout(x, 0.3, 9, site=10, site_dev=site, out=y)
            site.add_(1)
        for k in range(4):
            y.zero_()
            g.replay()
            s.synchronize()
            check_dropout(y, host(x), kept(64, 96, 0.3, 9, 10 + k), 0.3, "f32")
            x.add_(0.5)
            s.synchronize()
        c.close()


# ------------------------------------------------------------------ recurrence


def sigmoid(g):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))


class Seqs:
    """Inputs of a recurrence in a format, and their values in 64 bits."""

    def __init__(self, dtype, lengths, D, group=1, sig=True, state=True, seed=0, gate=None):
        rng = np.random.default_rng([seed, D, len(lengths)])
        self.dtype, self.D, self.group, self.sig, self.nseq = dtype, D, group, sig, len(lengths)
        self.off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
        n = self.n = int(self.off[-1])
        if gate is None:
            gate = rng.normal(1.5, 2.0, (n, D // group)) if sig else \
                rng.uniform(-0.2, 1.0, (n, D // group))
        self.gate = dev(gate, dtype)
        self.x, self.dh = dev(rng.normal(size=(n, D)), dtype), dev(rng.normal(size=(n, D)), dtype)
        self.h0 = dev(rng.normal(size=(self.nseq, D))) if state else None
        self.dlast = dev(rng.normal(size=(self.nseq, D))) if state else None

    def offsets(self, idt=torch.int32):
        return torch.from_numpy(self.off).to(idt).cuda()

    def decays(self):
        g = np.repeat(host(self.gate), self.group, 1)
        a, rest = sigmoid(g) if self.sig else (g, np.ones_like(g))
        # roundings of a decay and of its product: exp's argument, exp, the sum, the
        # reciprocal, 1 - a's own, the products and the sum of a token
        c = (np.abs(np.where(np.isfinite(g), g, 0)) if self.sig else 0 * g) + 12
        return a, rest, c * EPS

    def order(self, s, reverse):
        t = np.arange(self.off[s], self.off[s + 1])
        return t[::-1] if reverse else t

    def forward(self, reverse=False):
        """h, last and their bounds.  A part's error enters with the product of the decays
        that it goes through, whatever the order of the sums: E_t = a E_{t-1} + c eps H_t,
        with H the state of the absolute values."""
        a, rest, c = self.decays()
        x = host(self.x)
        h, E = np.zeros_like(x), np.zeros_like(x)
        last, lE = np.zeros((self.nseq, self.D)), np.zeros((self.nseq, self.D))
        for s in range(self.nseq):
            v = np.zeros(self.D) if self.h0 is None else host(self.h0[s])
            H, e = np.abs(v), 0.0
            for t in self.order(s, reverse):
                v = a[t] * v + rest[t] * x[t]
                H = np.abs(a[t]) * H + np.abs(rest[t] * x[t])
                e = np.abs(a[t]) * e + c[t] * H
                h[t], E[t] = v, e
            last[s], lE[s] = v, e
        return h, E, last, lE

    def backward(self, h, reverse=False):
        a, rest, c = self.decays()
        x, dh = host(self.x), host(self.dh)
        dx, dg = np.zeros_like(x), np.zeros_like(x)
        Ex, Eg, size = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
        dh0, E0 = np.zeros((self.nseq, self.D)), np.zeros((self.nseq, self.D))
        for s in range(self.nseq):
            mu = np.zeros(self.D) if self.dlast is None else host(self.dlast[s])
            start = np.zeros(self.D) if self.h0 is None else host(self.h0[s])
            H, e = np.abs(mu), 0.0
            o = self.order(s, reverse)
            for k in range(len(o) - 1, -1, -1):
                t = o[k]
                lam, L = dh[t] + mu, np.abs(dh[t]) + H
                before = h[o[k - 1]] if k else start
                el = e + 2 * EPS * L
                dx[t] = rest[t] * lam
                Ex[t] = rest[t] * el + c[t] * rest[t] * L
                w = before - x[t] if self.sig else before
                size[t] = np.abs(before) + (np.abs(x[t]) if self.sig else 0)
                f = a[t] * rest[t] if self.sig else np.ones(self.D)
                dg[t] = f * lam * w
                Eg[t] = f * (el * size[t] + (2 * c[t] + 4 * EPS) * L * size[t])
                size[t] = f * L * size[t]
                mu = a[t] * lam
                H = np.abs(a[t]) * L
                e = np.abs(a[t]) * el + c[t] * H
            dh0[s], E0[s] = mu, e
        shape = (self.n, self.D // self.group, self.group)
        dg, Eg, size = (v.reshape(shape).sum(2) for v in (dg, Eg, size))
        return dg, Eg + self.group * EPS * size, dx, Ex, dh0, E0

    def check(self, ctx, pg, reverse=False, idt=torch.int32, uniform=None, change=lambda t: t):
        form = pg.GATE_SIGMOID if self.sig else pg.GATE_RAW
        u, tiny = U[self.dtype], TINY[self.dtype]
        off = None if uniform else self.offsets(idt)

        def shape(t):
            t = change(t)
            return t.view(*uniform, -1) if uniform else t

        gate, x, dh = shape(self.gate), shape(self.x), shape(self.dh)
        h, last = ctx.recurrence(gate, x, off, h0=self.h0, form=form, reverse=reverse)
        assert h.shape == x.shape and last.dtype == torch.float32
        ref, E, rl, lE = self.forward(reverse)
        near(host(h).reshape(ref.shape), ref, E + u * (np.abs(ref) + E) + tiny, "h")
        near(host(last), rl, lE + EPS * np.abs(rl) + 1e-44, "last")
        dg, dx, dh0 = ctx.recurrence_backward(gate, x, shape(h.reshape(self.n, self.D)), dh, off,
                                              h0=self.h0, dlast=self.dlast, form=form,
                                              reverse=reverse)
        rg, Eg, rx, Ex, r0, E0 = self.backward(host(h).reshape(self.n, self.D), reverse)
        near(host(dx).reshape(rx.shape), rx, Ex + u * (np.abs(rx) + Ex) + tiny, "dx")
        near(host(dg).reshape(rg.shape), rg, Eg + u * (np.abs(rg) + Eg) + tiny, "dgate")
        if self.h0 is None:
            assert dh0 is None
        else:
            near(host(dh0), r0, E0 + EPS * np.abs(r0) + 1e-44, "dh0")
        assert ctx.status() == pg.OK
        return h, last, dg, dx, dh0


def some_lengths(rng, nseq, mean):
    n = rng.geometric(1.0 / (mean + 1), nseq) - 1
    return n if n.sum() else n + 1


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("sig", [True, False])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("D", [1, 5, 64, 130, 256, 300])
def test_recurrence_of_sentences(pg, ctx, dtype, sig, reverse, D):
    lengths = some_lengths(np.random.default_rng(D), 40, 14)
    Seqs(dtype, lengths, D, 1, sig, state=D != 64, seed=1).check(
        ctx, pg, reverse, torch.int64 if D % 2 else torch.int32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sig", [True, False])
@pytest.mark.parametrize("D,group", [(2, 2), (6, 3), (64, 16), (96, 32), (96, 48), (200, 100),
                                     (512, 128), (256, 256), (35, 5), (254, 127), (510, 255), (1024, 64)])
def test_recurrence_with_shared_gates(pg, ctx, dtype, sig, D, group):
    lengths = some_lengths(np.random.default_rng(group), 9, 25)
    Seqs(dtype, lengths, D, group, sig, seed=2).check(ctx, pg, group % 2 == 1)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("D,group", [(3, 1), (64, 1), (64, 16), (260, 1)])
@pytest.mark.parametrize("reverse", [False, True])
def test_recurrence_of_long_sequences(pg, ctx, dtype, D, group, reverse):
    """Longer than any part that a workgroup takes, alone and beside others."""
    Seqs(dtype, [3001], D, group, True, seed=3).check(ctx, pg, reverse)
    Seqs(dtype, [1, 1500, 0, 2, 777, 64, 128, 0], D, group, False, seed=4).check(ctx, pg, reverse)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("sig", [True, False])
@pytest.mark.parametrize("D,group", [(512, 1), (509, 1), (512, 64), (1020, 255)])
def test_recurrence_of_many_tokens(pg, ctx, dtype, sig, D, group):
    """Enough workgroups for the long chunks: sequences that begin and end in every place
    of them, and one that goes through many."""
    rng = np.random.default_rng(D + group)
    lengths = np.concatenate([rng.integers(0, 40, 30), [3200], rng.integers(100, 300, 6), [0, 1]])
    Seqs(dtype, np.append(lengths, 6001 - lengths.sum()), D, group, sig, state=sig,
         seed=25).check(ctx, pg, not sig)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256,
                               257, 511, 513])
def test_recurrence_of_every_length(pg, ctx, n):
    Seqs("f32", [n], 72, 1, True, seed=5).check(ctx, pg)
    Seqs("f32", [n, n, n], 24, 8, False, seed=6).check(ctx, pg, True, uniform=(3, n))


def test_recurrence_of_empty_sequences(pg, ctx):
    for lengths in ([0, 0, 3, 0, 0, 0, 64, 0, 0], [0] * 300 + [5] + [0] * 300, [0, 0, 0]):
        for state in (True, False):
            for reverse in (False, True):
                q = Seqs("f32", lengths, 36, 1, True, state=state, seed=7)
                q.check(ctx, pg, reverse)
    q = Seqs("bf16", [0, 0], 36, 1, True, seed=7)
    h, last, dg, dx, dh0 = q.check(ctx, pg)
    assert torch.equal(last, q.h0) and torch.equal(dh0, q.dlast) and h.numel() == 0


def test_recurrence_of_many_short_sequences(pg, ctx):
    rng = np.random.default_rng(8)
    Seqs("f32", rng.integers(0, 3, 4000), 20, 4, True, seed=8).check(ctx, pg)
    Seqs("f16", np.ones(3000, int), 20, 1, True, seed=9).check(ctx, pg, True, torch.int64)


def test_recurrence_of_equal_lengths(pg, ctx):
    for n, T in ((1, 1), (7, 1), (1, 300), (50, 3), (3, 130)):
        Seqs("bf16", [T] * n, 64, 1, True, seed=10).check(ctx, pg, n == 7, uniform=(n, T))
    q = Seqs("f32", [70], 64, 1, True, state=False)
    h, last = ctx.recurrence(q.gate, q.x)  # one sequence, no state
    near(host(h), q.forward()[0], q.forward()[1] * 2)


@pytest.mark.parametrize("dtype", list(DT))
def test_recurrence_strides(pg, ctx, dtype):
    """The halves of one projection, rows apart and starts that no vector is aligned to."""
    for D, group in ((64, 1), (64, 16), (61, 1)):
        q = Seqs(dtype, [40, 0, 90, 33], D, group, True, seed=11)
        q.check(ctx, pg, False, change=lambda t: strided(t, 3, 1))
        q.check(ctx, pg, True, change=lambda t: strided(t, 8, 8))
        both = torch.cat([q.x, q.dh], 1)
        a = ctx.recurrence(q.gate, both[:, :D], q.offsets(), h0=q.h0)[0]
        assert torch.equal(a, ctx.recurrence(q.gate, q.x, q.offsets(), h0=q.h0)[0])
        wide = torch.full((q.n, 2 * D + 1), 5.0, dtype=DT[dtype], device="cuda")
        ctx.recurrence(q.gate, q.x, q.offsets(), h0=q.h0, out=wide[:, D:2 * D])
        assert torch.equal(wide[:, D:2 * D], a)
        assert (wide[:, :D] == 5).all() and (wide[:, 2 * D:] == 5).all()


def test_recurrence_in_place(pg, ctx):
    q = Seqs("f32", [100, 0, 300], 64, 1, True, seed=12)
    off = q.offsets()
    h, last = ctx.recurrence(q.gate, q.x, off, h0=q.h0)
    s, x = q.h0.clone(), q.x.clone()
    ctx.recurrence(q.gate, x, off, h0=s, last=s, out=x)
    assert torch.equal(s, last) and torch.equal(x, h)
    dg, dx, dh0 = ctx.recurrence_backward(q.gate, q.x, h, q.dh, off, h0=q.h0, dlast=q.dlast)
    for name in ("dh", "x"):
        t, e = {"dh": q.dh.clone(), "x": q.x.clone()}, q.dlast.clone()
        r = ctx.recurrence_backward(q.gate, t["x"], h, t["dh"], off, h0=q.h0, dlast=e, dh0=e,
                                    dx=t[name])
        assert torch.equal(r[0], dg) and torch.equal(t[name], dx) and torch.equal(e, dh0)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("nseq,D,group", [(1, 1, 1), (3, 64, 1), (64, 256, 1), (5, 100, 100),
                                          (17, 130, 13), (2000, 24, 1)])
@pytest.mark.parametrize("sig", [True, False])
def test_recurrence_step(pg, ctx, dtype, nseq, D, group, sig):
    q = Seqs(dtype, [1] * nseq, D, group, sig, seed=13)
    form = pg.GATE_SIGMOID if sig else pg.GATE_RAW
    h, last = ctx.recurrence_step(q.gate, q.x, q.h0, form=form)
    ref, E, rl, lE = q.forward()
    near(host(h), ref, E + U[dtype] * (np.abs(ref) + E) + TINY[dtype])
    near(host(last), rl, lE)
    s = q.h0.clone()
    h2, s2 = ctx.recurrence_step(strided(q.gate, 1, 1), strided(q.x, 3, 1), s, form=form, last=s)
    assert s2 is s and torch.equal(s, last) and torch.equal(h2, h)
    h3, _ = ctx.recurrence_step(q.gate, q.x, form=form)  # from zeros
    q.h0 = None
    ref, E = q.forward()[:2]
    near(host(h3), ref, E + U[dtype] * (np.abs(ref) + E) + TINY[dtype])


def test_recurrence_steps_follow_the_whole(pg, ctx):
    """Token after token gives what the scan over all tokens gives."""
    q = Seqs("f32", [50] * 3, 40, 1, True, seed=14)
    ref, E, rl, lE = q.forward()
    s = q.h0.clone()
    gate, x = q.gate.view(3, 50, -1), q.x.view(3, 50, -1)
    for t in range(50):
        h, _ = ctx.recurrence_step(gate[:, t], x[:, t], s, last=s)
        near(host(h), ref.reshape(3, 50, -1)[:, t], E.reshape(3, 50, -1)[:, t] * 1.01)
    near(host(s), rl, lE * 1.01)


@pytest.mark.parametrize("reverse", [False, True])
def test_recurrence_keeps_sequences_apart(pg, ctx, reverse):
    """Values that are not finite stay in their sequence and channel."""
    lengths = [30, 200, 1, 64, 100]
    q = Seqs("f32", lengths, 40, 1, True, seed=15)
    off = q.offsets()
    h, last = ctx.recurrence(q.gate, q.x, off, h0=q.h0, reverse=reverse)
    dg, dx, dh0 = ctx.recurrence_backward(q.gate, q.x, h, q.dh, off, h0=q.h0, dlast=q.dlast,
                                          reverse=reverse)
    for bad in (math.nan, math.inf):
        x, d, s0, e0 = q.x.clone(), q.dh.clone(), q.h0.clone(), q.dlast.clone()
        x[40, 7] = bad    # sequence 1
        d[235, 9] = bad   # sequence 3
        s0[4, 3] = bad
        e0[0, 5] = bad
        h2, last2 = ctx.recurrence(q.gate, x, off, h0=s0, reverse=reverse)
        clean = torch.ones_like(h, dtype=torch.bool)
        clean[30:230, 7] = False
        clean[295:395, 3] = False
        assert torch.equal(h2[clean], h[clean])
        assert not torch.isfinite(h2[229 if not reverse else 30, 7])
        assert torch.isfinite(last2).sum() == last2.numel() - 2
        dg2, dx2, dh02 = ctx.recurrence_backward(q.gate, q.x, h, d, off, h0=q.h0, dlast=e0,
                                                 reverse=reverse)
        clean = torch.ones_like(h, dtype=torch.bool)
        clean[231:295, 9] = False
        clean[0:30, 5] = False
        assert torch.equal(dx2[clean], dx[clean]) and torch.equal(dg2[clean], dg[clean])


def test_recurrence_gates_at_their_limits(pg, ctx):
    n, D = 300, 8
    gate = np.zeros((n, D))
    gate[:, 0], gate[:, 1], gate[:, 2], gate[:, 3] = 100, -100, np.inf, -np.inf
    gate[:, 4], gate[:, 5] = 20, -20
    Seqs("f32", [n], D, 1, True, seed=16, gate=gate).check(ctx, pg)
    raw = np.zeros((n, D))
    raw[:, 0], raw[:, 1], raw[:, 2], raw[:, 3], raw[:, 4] = 1, 0, -1, 1e-30, 0.999
    Seqs("f32", [n], D, 1, False, seed=17, gate=raw).check(ctx, pg)


def test_recurrence_gradient_by_differences(pg, ctx):
    """sum(w h) + sum(v last) against central differences of the forward pass."""
    for sig, group, reverse in ((True, 1, False), (True, 4, True), (False, 1, True),
                                (False, 4, False)):
        form = pg.GATE_SIGMOID if sig else pg.GATE_RAW
        q = Seqs("f32", [5, 0, 70, 1], 8, group, sig, seed=18)
        off = q.offsets()
        h, _ = ctx.recurrence(q.gate, q.x, off, h0=q.h0, form=form, reverse=reverse)
        grads = ctx.recurrence_backward(q.gate, q.x, h, q.dh, off, h0=q.h0, dlast=q.dlast,
                                        form=form, reverse=reverse)
        rng = np.random.default_rng(19)

        def loss(gate, x, h0):
            h, last = ctx.recurrence(gate, x, off, h0=h0, form=form, reverse=reverse)
            return float((h.double() * q.dh.double()).sum()
                         + (last.double() * q.dlast.double()).sum())

        args = [q.gate, q.x, q.h0]
        _, E, _, lE = q.forward(reverse)
        off_by = (np.abs(host(q.dh)) * (E + EPS)).sum() + (np.abs(host(q.dlast)) * (lE + EPS)).sum()
        step = 2.0 ** -4

        def difference(k, v, step):
            up, down = list(args), list(args)
            up[k], down[k] = args[k] + step * v, args[k] - step * v
            return (loss(*up) - loss(*down)) / (2 * step)

        for k in range(3):
            for _ in range(3):
                v = dev(rng.choice([-1.0, 1.0], size=tuple(args[k].shape)))
                d1, d2 = difference(k, v, step), difference(k, v, step / 2)
                want = float((grads[k].double() * v.double()).sum())
                # extrapolated to a step of zero; what remains is below the two steps' own
                # difference, beside the forward passes' roundings over the steps
                tol = abs(d1 - d2) + 3 * off_by / step + 1e-5 * abs(want)
                assert abs((4 * d2 - d1) / 3 - want) <= tol, (sig, group, reverse, k)


def test_recurrence_results_do_not_depend_on_the_run(pg, ctx):
    q = Seqs("f32", [2000, 1, 3000, 500], 96, 32, True, seed=20)
    first = q.check(ctx, pg)
    for _ in range(5):
        h, last = ctx.recurrence(q.gate, q.x, q.offsets(), h0=q.h0)
        assert torch.equal(h, first[0]) and torch.equal(last, first[1])
        r = ctx.recurrence_backward(q.gate, q.x, h, q.dh, q.offsets(), h0=q.h0, dlast=q.dlast)
        assert all(torch.equal(a, b) for a, b in zip(r, first[2:]))


def test_recurrence_widths_take_turns(pg):
    """Calls that cut their channels into other numbers of tiles share one workspace: what
    an earlier call left in it must not be taken for this call's."""
    c = pg.Context(1000, 16, 5, 8, max_batch=1)
    c.reserve_recurrence(3000, 1100)
    qs = [Seqs("f32", [2500, 0, 400], D, g, True, seed=D) for D, g in
          ((64, 1), (1024, 1), (8, 1), (520, 2), (1100, 1))]
    ref = [q.forward() for q in qs]
    for _ in range(3):
        for k in (0, 0, 1, 2, 3, 0, 4, 1, 2, 4, 3):
            h, E, last, lE = ref[k]
            got = c.recurrence(qs[k].gate, qs[k].x, qs[k].offsets(), h0=qs[k].h0)
            near(host(got[0]), h, E + EPS * np.abs(h), k)
            near(host(got[1]), last, lE + EPS * np.abs(last), k)
    c.close()


def test_recurrence_in_a_graph(pg):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = pg.Context(1000, 16, 5, 8, max_batch=1, stream=s)
        c.reserve_recurrence(4000, 64)
        q = Seqs("f32", [1500, 0, 900], 64, 1, True, seed=21)
        off, h, last = q.offsets(), torch.empty_like(q.x), torch.empty_like(q.h0)
        dg, dx, dh0 = torch.empty_like(q.x), torch.empty_like(q.x), torch.empty_like(q.h0)

        def both():
            c.recurrence(q.gate, q.x, off, h0=q.h0, out=h, last=last)
            c.recurrence_backward(q.gate, q.x, h, q.dh, off, h0=q.h0, dlast=q.dlast, dgate=dg,
                                  dx=dx, dh0=dh0)

        both()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            both()
        outs = (h, last, dg, dx, dh0)
        for k in range(4):
            for t in outs:
                t.zero_()
            g.replay()
            s.synchronize()
            got = [t.clone() for t in outs]
            both()
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, outs)), k
            q.x.mul_(1.25)
            s.synchronize()
        c.close()


def test_recurrence_offsets_that_do_not_ascend(pg, ctx):
    q = Seqs("f32", [10, 20, 30], 16, 1, True, seed=22)
    for off in ([0, 30, 10, 60], [1, 10, 30, 60], [0, 10, 30, 59], [0, 10, 30, 61],
                [-5, 10, 30, 60], [0, 1 << 40, 30, 60]):
        t = torch.tensor(off, dtype=torch.int64, device="cuda")
        h, _ = ctx.recurrence(q.gate, q.x, t, h0=q.h0)
        assert ctx.status() == pg.EOFFSETS
        ctx.recurrence_backward(q.gate, q.x, q.x, q.dh, t, h0=q.h0)
        assert ctx.status() == pg.EOFFSETS
    q.check(ctx, pg)


def test_recurrence_rows_past_32_bits(pg, ctx):
    ld = (1 << 31) + 1024
    buf = torch.empty(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    q = Seqs("bf16", [3], 48, 1, True, seed=23)
    x = buf.as_strided((3, 48), (ld, 1))
    x.copy_(q.x)
    a = ctx.recurrence(q.gate, q.x, q.offsets(), h0=q.h0)[0]
    assert torch.equal(ctx.recurrence(q.gate, x, q.offsets(), h0=q.h0)[0], a)
    ctx.recurrence(q.gate, x, q.offsets(), h0=q.h0, out=x)
    assert torch.equal(x, a)


# ------------------------------------------------------------------ scores


def logits_ref(l, V, hist, rep, freq, pres, bias, allowed):
    """One row in 64 bits: the scores, and the size of what was rounded for each."""
    l = l.copy()
    size = np.abs(l)
    if hist is not None:
        ids, made = hist
        u = np.unique(ids[(ids >= 0) & (ids < V)])
        l[u] = np.where(l[u] > 0, l[u] / rep, l[u] * rep)
        size[u] = np.abs(l[u])
        u, n = np.unique(made[(made >= 0) & (made < V)], return_counts=True)
        l[u] -= freq * n + pres
        size[u] += 2 * (np.abs(freq * n) + abs(pres))
    if bias is not None:
        l += bias
        size += np.abs(bias)
    if allowed is not None:
        l[~allowed] = -np.inf
    return l, size


class Scores:
    def __init__(self, dtype, rows, V, cap=0, masks=None, bias=None, seed=0):
        rng = np.random.default_rng([seed, rows, V])
        self.dtype, self.rows, self.V, self.cap = dtype, rows, V, cap
        self.logits = dev(rng.normal(0, 3, (rows, V)), dtype)
        self.kw = {}
        if cap:
            hist = np.minimum((np.exp(rng.uniform(0, np.log(V + 1), (rows, cap))) - 1), V - 1)
            hist = np.where(rng.random((rows, cap)) < 0.05, -1, hist).astype(np.int32)
            length = rng.integers(0, cap + 1, rows)
            length[0] = cap
            self.kw.update(
                history=torch.from_numpy(hist).cuda(),
                lengths=torch.from_numpy(length.astype(np.int32)).cuda(),
                prompt=torch.from_numpy((length * rng.random(rows)).astype(np.int32)).cuda(),
                repetition=dev(rng.uniform(0.8, 1.5, rows)), presence=dev(rng.uniform(-1, 1, rows)),
                frequency=dev(rng.uniform(0, 0.5, rows)))
        if bias:
            self.kw["bias"] = dev(rng.normal(size=(rows, V) if bias == "rows" else V))
        if masks is not None:
            bits = rng.random((masks, V)) < rng.uniform(0, 1, (masks, 1))
            self.set_mask(bits)
            if masks not in (1, rows):
                self.kw["mask_rows"] = torch.from_numpy(
                    rng.integers(-1, masks, rows).astype(np.int32)).cuda()

    def set_mask(self, bits):
        n, V = bits.shape
        self.bits = bits
        full = np.zeros((n, (V + 31) // 32 * 32), bool)
        full[:, :V] = bits
        words = np.packbits(full, axis=1, bitorder="little").view(np.uint32)
        self.kw["mask"] = torch.from_numpy(words.view(np.int32).copy()).cuda()

    def reference(self):
        kw = {k: v.cpu().numpy() for k, v in self.kw.items()}
        l = host(self.logits)
        out, size = np.empty_like(l), np.empty_like(l)
        for r in range(self.rows):
            hist = None
            if "history" in kw:
                n = min(max(kw["lengths"][r], 0), self.cap) if "lengths" in kw else self.cap
                k = min(max(kw["prompt"][r], 0), self.cap) if "prompt" in kw else 0
                hist = kw["history"][r, :n], kw["history"][r, k:n]
            bias = kw.get("bias")
            bias = None if bias is None else (bias if bias.ndim == 1 else bias[r]).astype(float)
            allowed = None
            if "mask" in kw:
                m = kw["mask_rows"][r] if "mask_rows" in kw else (r if len(self.bits) > 1 else 0)
                allowed = self.bits[m] if 0 <= m < len(self.bits) else None
            one = lambda name, v: float(kw[name][r]) if name in kw else v  # noqa: E731
            out[r], size[r] = logits_ref(l[r], self.V, hist, one("repetition", 1.0),
                                         one("frequency", 0.0), one("presence", 0.0), bias, allowed)
        return out, size

    def check(self, ctx, got=None, logits=None):
        """The scores' own bound, then the choice and the log-sum-exp by theirs."""
        out, token, lse = got or ctx.logits(self.logits if logits is None else logits, **self.kw)
        ref, size = self.reference()
        E = 6 * EPS * size
        if out is not None:
            fin = np.isfinite(ref)
            g = host(out)
            assert np.array_equal(g == -np.inf, ref == -np.inf)
            near(np.where(fin, g, 0), np.where(fin, ref, 0),
                 E + U[self.dtype] * (np.abs(np.where(fin, ref, 0)) + E) + TINY[self.dtype], "out")
        t, z = token.cpu().numpy(), host(lse)
        for r in range(self.rows):
            top = ref[r].max()
            if top == -np.inf:
                assert t[r] == -1 and z[r] == -np.inf
                continue
            assert ref[r, t[r]] + E[r, t[r]] >= top - E[r].max(), r
            want = top + np.log(np.exp(ref[r] - top).sum())
            # the scores' errors; a sum of V terms, each with its exponential's error of an
            # argument below 110 (smaller terms vanish); the logarithm and the last sum
            bound = E[r].max() + (self.V / 64 + 64 + 110) * EPS + 4 * EPS * (abs(top) + abs(want))
            assert abs(z[r] - want) <= bound, (r, z[r], want, bound)
        return out, token, lse


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (4, 3), (1, 4), (2, 5), (2, 31), (3, 32), (5, 33), (1, 1000), (4, 4099),
                                    (2, 8191), (2, 8192), (3, 8193), (2, 32003), (33, 2047),
                                    (1, 100_000)])
def test_scores(ctx, dtype, rows, V):
    Scores(dtype, rows, V).check(ctx)
    Scores(dtype, rows, V, cap=50, masks=rows, bias="shared", seed=1).check(ctx)
    Scores(dtype, rows, V, cap=7, masks=1, bias="rows", seed=2).check(ctx)
    Scores(dtype, rows, V, cap=300, masks=rows + 2, seed=3).check(ctx)


@pytest.mark.parametrize("cap", [1, 255, 256, 257, 2047, 2049, 5000, 20_000, 32_767, 32_768,
                                 50_000])
def test_scores_with_histories(ctx, cap):
    q = Scores("f32", 3, 9001, cap=cap, seed=4)
    q.check(ctx)
    del q.kw["lengths"]  # the whole of each row
    q.check(ctx)
    del q.kw["prompt"]  # all of it made by the model
    q.check(ctx)
    q.kw["lengths"] = torch.tensor([-3, 0, cap + 9], dtype=torch.int32, device="cuda")
    q.kw["prompt"] = torch.tensor([5, cap + 4, -7], dtype=torch.int32, device="cuda")
    q.check(ctx)
    del q.kw["repetition"], q.kw["presence"], q.kw["frequency"]  # nothing to apply
    out = q.check(ctx)[0]
    assert torch.equal(out, q.logits)


@pytest.mark.parametrize("cap", [6000, 32_767, 70_000])
def test_scores_of_one_word_many_times(ctx, cap):
    q = Scores("f32", 2, 500, cap=cap, seed=5)
    q.kw["history"].fill_(17)
    q.kw["history"][:, ::2] = 499
    q.check(ctx)


@pytest.mark.parametrize("dtype", list(DT))
def test_scores_forms_of_the_output(ctx, dtype):
    q = Scores(dtype, 6, 5003, cap=40, masks=6, bias="shared", seed=6)
    out, token, lse = q.check(ctx)
    none, t2, l2 = ctx.logits(q.logits, write=False, **q.kw)
    assert none is None and torch.equal(t2, token) and torch.equal(l2, lse)
    z = q.logits.clone()
    o3, t3, l3 = ctx.logits(z, out=z, **q.kw)
    assert o3 is z and torch.equal(z, out) and torch.equal(t3, token) and torch.equal(l3, lse)
    for pad, shift in ((3, 1), (8, 8), (13, 2)):
        o = strided(torch.zeros_like(z), pad, shift)
        guard = o._base.clone()
        o4, t4, l4 = ctx.logits(strided(q.logits, pad, shift), out=o, **q.kw)
        assert torch.equal(o4, out) and torch.equal(t4, token)
        near(host(l4), host(lse), 2 * (q.V / 64 + 200) * EPS)
        o.zero_()
        assert torch.equal(o._base, guard)


def test_scores_ties_go_to_the_lowest_word(ctx):
    for V in (40, 3000, 70_001):
        x = torch.zeros(5, V, device="cuda")
        x[1, V - 1] = x[1, V // 2] = 2.0
        x[2, V - 1] = 1.0
        x[3, :] = -math.inf
        x[3, V // 3:] = -5.0
        x[4, :] = torch.finfo(torch.float32).min
        token = ctx.logits(x)[1].tolist()
        assert token == [0, V // 2, V - 1, V // 3, 0]
        h = ctx.logits(x.half(), bias=torch.zeros(V, device="cuda"))[1].tolist()
        assert h == [0, V // 2, V - 1, V // 3, -1]  # float16 holds the lowest float as -infinity


def test_scores_that_are_not_finite(ctx):
    V = 9000
    x = torch.randn(7, V, device="cuda")
    bits = np.ones((7, V), bool)
    x[0, 100], bits[0, 100] = math.nan, False        # not a number where the mask is
    x[1, 8999], bits[1, 8999] = math.inf, False
    x[2, 5] = math.inf
    x[2, 4000] = math.inf
    x[3, 50] = math.nan
    x[4, :] = -math.inf
    bits[5] = False                                   # nothing allowed
    x[6, :] = math.nan
    q = Scores("f32", 7, V, seed=7)
    q.logits = x
    q.set_mask(bits)
    out, token, lse = ctx.logits(x, **q.kw)
    o, z, t = host(out), host(lse), token.tolist()
    ref = np.where(bits, host(x), -np.inf)
    assert np.array_equal(o, ref, equal_nan=True)
    assert t[0] == int(np.argmax(ref[0])) and t[1] == int(np.argmax(ref[1]))
    assert np.isfinite(z[:2]).all()
    assert t[2] == 5 and z[2] == math.inf
    assert t[3] == int(np.nanargmax(ref[3])) and math.isnan(z[3])
    assert t[4] == -1 and z[4] == -math.inf
    assert t[5] == -1 and z[5] == -math.inf
    assert t[6] == -1 and math.isnan(z[6])


def test_scores_far_apart(ctx):
    """Masks of the type's lowest value and scores that a plain sum of exponentials overflows."""
    for dtype in DT:
        low = torch.finfo(DT[dtype]).min
        x = torch.full((3, 5000), low, dtype=DT[dtype], device="cuda")
        x[0, 4321] = 3.0
        x[1, :] = 60000.0
        x[2, 9] = -60000.0
        out, token, lse = ctx.logits(x)
        assert torch.equal(out, x)
        assert token.tolist()[:2] == [4321, 0]
        z = host(lse)
        assert z[0] == 3.0
        top = float(x[1, 0])
        assert abs(z[1] - (top + math.log(5000))) <= 4 * EPS * top
        assert math.isfinite(z[2])


def test_scores_with_bad_ids(pg, ctx):
    q = Scores("f32", 3, 700, cap=20, masks=5, seed=8)
    ref = ctx.logits(q.logits, **q.kw)
    kw = dict(q.kw, history=q.kw["history"].clone(), lengths=torch.full_like(q.kw["lengths"], 20))
    kw["history"][1, 3] = -9
    want = ctx.logits(q.logits, **kw)[0]
    assert ctx.status() == pg.OK
    kw["history"][1, 3] = 700
    got = ctx.logits(q.logits, **kw)[0]
    assert ctx.status() == pg.EID and torch.equal(got, want)
    kw = dict(q.kw, mask_rows=torch.tensor([0, 5, -1], dtype=torch.int32, device="cuda"))
    free = ctx.logits(q.logits, **dict(q.kw, mask_rows=torch.tensor(
        [0, -1, -1], dtype=torch.int32, device="cuda")))
    assert ctx.status() == pg.OK
    got = ctx.logits(q.logits, **kw)
    assert ctx.status() == pg.EID
    assert all(torch.equal(a, b) for a, b in zip(got, free))
    assert all(torch.equal(a, b) for a, b in zip(ref, ctx.logits(q.logits, **q.kw)))


def test_scores_of_many_rows(ctx):
    """Enough rows for the longest parts, in every format."""
    for dtype in DT:
        q = Scores(dtype, 64, 70_003, cap=300, masks=64, bias="shared", seed=12)
        q.check(ctx)


def test_scores_in_a_graph(pg):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = pg.Context(1000, 16, 5, 8, max_batch=1, stream=s)
        c.reserve_logits(4, 50_000)
        q = Scores("bf16", 4, 50_000, cap=100, masks=4, seed=9)
        c.logits(q.logits, **q.kw)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got = c.logits(q.logits, **q.kw)
        for k in range(4):
            for t in got:
                t.zero_()
            g.replay()
            s.synchronize()
            want = c.logits(q.logits, **q.kw)
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), k
            q.logits.copy_(torch.randn_like(q.logits.float()))
            s.synchronize()
        c.close()


def test_scores_do_not_depend_on_the_run(ctx):
    q = Scores("f32", 9, 60_007, cap=500, masks=9, seed=10)
    first = q.check(ctx)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, ctx.logits(q.logits, **q.kw)))


def test_scores_rows_past_32_bits(ctx):
    ld = (1 << 32) + 640
    buf = torch.empty(ld + 5000, dtype=torch.float16, device="cuda")
    q = Scores("f16", 2, 4999, cap=9, masks=2, seed=11)
    x = buf.as_strided((2, 4999), (ld, 1))
    x.copy_(q.logits)
    q.check(ctx, ctx.logits(x, out=x, **q.kw))


# ------------------------------------------------------------------ refusals


def test_refusals(pg, ctx):
    """Bad arguments raise with their code and enqueue nothing."""
    x = torch.zeros(8, 16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")

    def refused(code, f):
        with pytest.raises(pg.PolyglotError) as e:
            f()
        assert e.value.rc == code

    for p in (-0.1, 1.1, math.nan):
        refused(pg.EINVAL, lambda: ctx.dropout(x, p, 1))
    refused(pg.EINVAL, lambda: ctx.dropout(x, 0.1, 1, ids=torch.zeros(8, **i32), out=x))
    for f in (lambda: ctx.dropout(x.double(), 0.1, 1), lambda: ctx.dropout(x, 0.1, 1, add=x.half()),
              lambda: ctx.dropout(x, 0.1, 1, ids=x[:, 0])):
        with pytest.raises(TypeError):
            f()
    for f in (lambda: ctx.dropout(x.cpu(), 0.1, 1), lambda: ctx.dropout(x.t(), 0.1, 1),
              lambda: ctx.dropout(x, 0.1, 1, out=torch.zeros(8, 15, device="cuda"))):
        with pytest.raises(ValueError):
            f()

    off = torch.tensor([0, 8], **i32)
    small = pg.Context(1000, 16, 5, 8, max_batch=1)
    refused(pg.EBATCH, lambda: small.recurrence(x, x, off))  # nothing reserved
    small.recurrence_step(x, x)                                # needs nothing
    small.reserve_recurrence(8, 15)
    refused(pg.EBATCH, lambda: small.recurrence(x, x, off))
    small.reserve_recurrence(7, 16)
    refused(pg.EBATCH, lambda: small.recurrence_backward(x, x, x, x, off))
    small.reserve_recurrence(8, 16)
    small.recurrence(x, x, off)
    refused(pg.EBATCH, lambda: small.logits(x))
    small.reserve_logits(8, 16)
    small.logits(x)
    refused(pg.EINVAL, lambda: small.reserve_recurrence(-1, 16))
    refused(pg.EINVAL, lambda: small.reserve_logits(8, -1))
    assert small.status() == pg.OK
    small.close()

    refused(pg.EINVAL, lambda: ctx.recurrence(x, x, off, form=2))
    refused(pg.EBATCH, lambda: ctx.recurrence(x, x, off[:1]))  # no sequence
    wide = torch.zeros(8, 514, device="cuda")
    refused(pg.EINVAL, lambda: ctx.recurrence(wide[:, :2].contiguous(), wide, off))  # 257 share a gate
    refused(pg.EINVAL, lambda: ctx.recurrence(x, torch.ones_like(x), off, out=x))
    h = torch.ones_like(x)
    refused(pg.EINVAL, lambda: ctx.recurrence_backward(x, x, h, x, off, dx=h))
    refused(pg.EINVAL, lambda: ctx.recurrence_backward(h, x, x, x, off, dgate=h))
    for f in (lambda: ctx.recurrence(x[:, :3], x, off), lambda: ctx.recurrence(x[:7], x, off),
              lambda: ctx.recurrence(x, x, off, h0=torch.zeros(2, 16, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ctx.recurrence(x.half(), x, off), lambda: ctx.recurrence(x, x, off.float()),
              lambda: ctx.recurrence(x, x, off, h0=torch.zeros(1, 16, device="cuda").half())):
        with pytest.raises(TypeError):
            f()

    mask = torch.zeros(3, 1, **i32)
    refused(pg.EINVAL, lambda: ctx.logits(x, mask=mask))  # three masks, eight rows, no mask_rows
    for f in (lambda: ctx.logits(x, mask=torch.zeros(8, 2, **i32)),
              lambda: ctx.logits(x, bias=torch.zeros(15, device="cuda")),
              lambda: ctx.logits(x, history=torch.zeros(7, 4, **i32)),
              lambda: ctx.logits(x, repetition=torch.ones(1, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ctx.logits(x.int()), lambda: ctx.logits(x, history=x.long()),
              lambda: ctx.logits(x, presence=torch.zeros(8, device="cuda").double())):
        with pytest.raises(TypeError):
            f()


def test_refusals_of_the_c_entries(pg, ctx):
    lib, h = pg.load_library(), ctx._h
    x = torch.zeros(64, device="cuda")
    p = x.data_ptr()
    d = dict(x=p, y=p, rows=2, ld_x=8, ld_y=8, d=8, p=0.5)
    ok = lambda cls, **kw: cls(**kw)  # noqa: E731
    call = lib.polyglot_dropout
    assert call(h, ctypes.byref(ok(pg.DropoutArgs, **d))) == pg.OK
    for change, code in ((dict(rows=-1), pg.EBATCH), (dict(d=0), pg.EINVAL),
                         (dict(dtype=3), pg.EINVAL), (dict(x=0), pg.ENULL), (dict(y=0), pg.ENULL),
                         (dict(ld_x=7), pg.EINVAL), (dict(ld_y=7), pg.EINVAL),
                         (dict(ld_y=9), pg.EINVAL), (dict(x=p + 2), pg.EINVAL),
                         (dict(ids=p, id_bytes=2, table_rows=4), pg.EINVAL),
                         (dict(ids=p, id_bytes=4, table_rows=0), pg.EINVAL),
                         (dict(ld_x=1 << 62, ld_y=1 << 62), pg.EINVAL), (dict(rows=0), pg.OK)):
        assert call(h, ctypes.byref(ok(pg.DropoutArgs, **dict(d, **change)))) == code, change
    r = dict(gate=p, x=p, h=p + 128, tokens=2, ld_gate=8, ld_x=8, ld_h=8, nseq=1, D=8, group=1)
    call = lib.polyglot_recurrence
    assert call(h, ctypes.byref(ok(pg.RecurrenceArgs, **r))) == pg.OK
    for change, code in ((dict(nseq=0), pg.EBATCH), (dict(tokens=-1), pg.EBATCH),
                         (dict(tokens=1 << 31), pg.EBATCH), (dict(tokens=3, nseq=2), pg.EINVAL),
                         (dict(group=3), pg.EINVAL), (dict(group=0), pg.EINVAL),
                         (dict(dtype=-1), pg.EINVAL), (dict(form=5), pg.EINVAL),
                         (dict(gate=0), pg.ENULL), (dict(x=0), pg.ENULL), (dict(h=0), pg.ENULL),
                         (dict(offsets=p, offset_bytes=2), pg.EINVAL),
                         (dict(offsets=p + 4, offset_bytes=8), pg.EINVAL),
                         (dict(h0=p + 1), pg.EINVAL), (dict(ld_h=7), pg.EINVAL)):
        assert call(h, ctypes.byref(ok(pg.RecurrenceArgs, **dict(r, **change)))) == code, change
    g = dict(gate=p, x=p, h=p, dh=p, dgate=p + 64, dx=p + 128, tokens=2, ld_gate=8, ld_x=8, ld_h=8,
             ld_dh=8, ld_dgate=8, ld_dx=8, nseq=1, D=8, group=1, form=1)
    call = lib.polyglot_recurrence_grad
    assert call(h, ctypes.byref(ok(pg.RecurrenceGradArgs, **g))) == pg.OK
    assert call(h, ctypes.byref(ok(pg.RecurrenceGradArgs, **dict(g, x=0, ld_x=0, form=0)))) == pg.OK
    for change, code in ((dict(x=0), pg.ENULL), (dict(dh=0), pg.ENULL), (dict(dgate=0), pg.ENULL),
                         (dict(dx=0), pg.ENULL), (dict(dh0=p + 2), pg.EINVAL),
                         (dict(dgate=p), pg.EINVAL), (dict(dgate=p + 128), pg.EINVAL)):
        assert call(h, ctypes.byref(ok(pg.RecurrenceGradArgs, **dict(g, **change)))) == code, change
    v = dict(logits=p, out=p + 128, token=p + 64, rows=2, V=8, ld_logits=8, ld_out=8)
    call = lib.polyglot_logits
    assert call(h, ctypes.byref(ok(pg.LogitsArgs, **v))) == pg.OK
    for change, code in ((dict(rows=-1), pg.EBATCH), (dict(V=0), pg.EINVAL),
                         (dict(history_cap=-1), pg.EINVAL), (dict(logits=0), pg.ENULL),
                         (dict(out=0, token=0), pg.ENULL), (dict(ld_out=7), pg.EINVAL),
                         (dict(mask=p, ld_mask=1), pg.EINVAL), (dict(bias=p, ld_bias=3), pg.EINVAL),
                         (dict(mask=p, masks=1, ld_mask=0), pg.EINVAL),
                         (dict(rows=65), pg.EBATCH), (dict(lse=p + 2), pg.EINVAL),
                         (dict(out=p, ld_out=9), pg.EINVAL), (dict(rows=0), pg.OK)):
        assert call(h, ctypes.byref(ok(pg.LogitsArgs, **dict(v, **change)))) == code, change
    for name in ("polyglot_dropout", "polyglot_recurrence", "polyglot_recurrence_grad",
                 "polyglot_logits"):
        assert getattr(lib, name)(None, None) == pg.ENULL and getattr(lib, name)(h, None) == pg.ENULL
    assert lib.polyglot_reserve_recurrence(None, 1, 1) == pg.ENULL
    assert lib.polyglot_reserve_logits(None, 1, 1) == pg.ENULL
    assert lib.polyglot_operator_times(None, None, None) == pg.ENULL
    torch.cuda.synchronize()


def test_operator_times(pg):
    c = pg.Context(1000, 16, 5, 8, max_batch=1)
    c.reserve_logits(4, 100)
    c.set_timing(True)
    x = torch.randn(4, 100, device="cuda")
    c.dropout(x, 0.1, 1)
    c.logits(x)
    t = c.operator_times()
    assert set(t) == set(pg.OPERATOR_NAMES)
    assert t["dropout"][1] == 1 and t["dropout"][0] > 0 and t["logits"][1] >= 1
    assert t["recurrence"][1] == 0
    c.dropout(x, 0.1, 1)
    assert all(n == 0 for _, n in c.kernel_times().values())  # the others' ids; ours are kept
    assert c.operator_times()["dropout"][1] == 1
    c.close()


def test_tensors_of_another_stream(pg):
    """A context on a stream of its own, with tensors that another stream made."""
    s = torch.cuda.Stream()
    c = pg.Context(1000, 16, 5, 8, max_batch=1, stream=s)
    c.reserve_recurrence(1000, 64)
    q = Seqs("f32", [600, 0, 400], 64, 1, True, seed=24)
    off = q.offsets()
    s.wait_stream(torch.cuda.current_stream())
    h = torch.empty_like(q.x)
    last = torch.empty_like(q.h0)
    s.wait_stream(torch.cuda.current_stream())
    c.recurrence(q.gate, q.x, off, h0=q.h0, out=h, last=last)
    torch.cuda.current_stream().wait_stream(s)
    ref, E, rl, lE = q.forward()
    near(host(h), ref, E + EPS * np.abs(ref))
    assert c.status() == pg.OK
    c.close()
