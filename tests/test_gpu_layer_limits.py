"""The selective layer and beam search at their limits: steps of no length and of any length,
sums that are exact, sizes that take every form of the kernels, calls without the reserved
workspace.  The operators' ordinary tests are in test_gpu_layers.py."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import layer_refs as ref  # noqa: E402
from test_gpu_layers import (DT, F32_OUT, check_scan, cuda, cuts, near, normal, scan_call,  # noqa: E402
                             scan_inputs, scan_reference, wide)


@pytest.fixture(scope="module")
def pg():
    import paper_1404_1521_amd as pg
    return pg


@pytest.fixture(scope="module")
def ctx(pg):
    c = pg.Context(1000, 16, 5, 8, max_batch=1)
    c.reserve_selective(70_000, 1100, 64)
    c.reserve_beam(512, 100_003, 64)
    yield c
    assert c.status() == pg.OK
    c.close()


# ------------------------------------------------------------------ steps


@pytest.mark.parametrize("dtype", list(DT))
def test_selective_steps_of_no_length(ctx, dtype):
    """A delta of -infinity, whose softplus is 0, leaves the state as it was: what the other
    tokens give is what they give without it, bit for bit, and every gradient is finite."""
    gen = torch.Generator().manual_seed(21)
    n, D, N = 14, 9, 8
    out = [0, 3, 4, 9, 13]  # the tokens left out: the first and the last among them
    keep = [t for t in range(n) if t not in out]
    s = scan_inputs(gen, n, D, N, 1, 1, dtype)
    s["delta"][out] = -math.inf
    o = torch.tensor([0, n], dtype=torch.int32).cuda()
    got = scan_call(ctx, s, o, True)
    for k, v in got.items():
        assert torch.isfinite(v).all(), k
    rows = ("x", "delta", "B", "C", "z", "dy")
    less = {k: v[keep].contiguous() if k in rows else v for k, v in s.items()}
    want = scan_call(ctx, less, torch.tensor([0, len(keep)], dtype=torch.int32).cuda(), True)
    at = torch.tensor(keep).cuda()
    assert torch.equal(got["y"][at], want["y"]) and torch.equal(got["last"], want["last"])
    assert not got["delta"][out].any() and not got["B"][out].any()
    # against the formulas, where a softplus of -200 is e^-200: nothing in 32 bits, and below
    # the least normal number nothing is promised
    far = {k: None if v is None else v.clone() for k, v in s.items()}
    far["delta"][out] = -200.0
    values, err = scan_reference(far, [0, n], True, 0)
    for k in err:
        err[k] = err[k] + 1e-36
    check_scan(got, values, err, dtype, "no length")
    # token by token
    c = {k: cuda(v) for k, v in s.items()}
    state = c["h0"]
    for t in range(n):
        row = lambda k: c[k][t:t + 1]
        y, new = ctx.selective_step(row("x"), row("delta"), c["A"], row("B"), row("C"), state, skip=c["skip"],
                                    z=row("z"), delta_bias=c["bias"])
        if t in out:
            assert torch.equal(new, state), t
        near(y, values["y"][t:t + 1], ref.rounded(err["y"][t:t + 1], values["y"][t:t + 1], dtype), t)
        state = new
    near(state, values["last"], ref.rounded(err["last"], values["last"], "f32"), "last")


def test_selective_steps_of_any_length(ctx):
    """A delta above half of the largest number is its own softplus: the state decays to
    nothing, and with x = 0 nothing comes in."""
    gen = torch.Generator().manual_seed(22)
    n, D, N = 6, 5, 16
    s = scan_inputs(gen, n, D, N, 1, 1, "f32", bias=False)
    s["delta"][2], s["x"][2] = 3e38, 0.0
    o = torch.tensor([0, n], dtype=torch.int32).cuda()
    got = scan_call(ctx, s, o, True)
    for k, v in got.items():
        if k != "x":  # (its gradient is the step times what comes back)
            assert torch.isfinite(v).all(), k
    tail = {k: v[3:].contiguous() if k in ("x", "delta", "B", "C", "z", "dy") else v for k, v in s.items()}
    tail["h0"] = torch.zeros_like(s["h0"])
    want = scan_call(ctx, tail, torch.tensor([0, n - 3], dtype=torch.int32).cuda(), True)
    assert torch.equal(got["y"][3:], want["y"]) and torch.equal(got["last"], want["last"])
    c = {k: cuda(v) for k, v in s.items()}
    _, new = ctx.selective_step(c["x"][2:3], c["delta"][2:3], c["A"], c["B"][2:3], c["C"][2:3], c["h0"])
    assert not new.any()


# ------------------------------------------------------------------ sizes


def test_selective_of_the_most_tokens(pg):
    """One sequence of 2^30 tokens whose steps are 0: the state at its end is the one before it,
    and so is the gradient, going back."""
    n = 1 << 30
    ctx = pg.Context(1000, 16, 5, 8, max_batch=1)
    ctx.reserve_selective(n, 1, 1)
    none = torch.zeros(n, 1, dtype=torch.bfloat16, device="cuda")  # every input is the same zeros
    A = -torch.ones(1, 1, device="cuda")
    h0 = torch.full((1, 1, 1), 3.0, device="cuda")
    ins = (none, none, A, none, none)
    y, last, marks = ctx.selective_scan(*ins, state=h0, softplus=False, marks=True)
    zero = not y.any().item()  # (a failure is to print no tensor of this size)
    assert zero and torch.equal(last, h0)
    del y
    g = ctx.selective_backward(*ins, none, marks, state=h0, dlast=h0 + 2, softplus=False)
    # ddelta is A times what comes back, 5, times the state before, 3
    right = [(g.delta == -15).all().item(), not g.x.any().item(), not g.C.any().item(), not g.A.any().item()]
    assert all(right) and torch.equal(g.state, h0 + 2), right
    assert ctx.status() == pg.OK
    ctx.close()
    del g, marks, none, ins
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ workspace


@pytest.mark.parametrize("D,N,groups", [(40, 16, 1), (64, 24, 2), (33, 4, 1), (20, 64, 1)])
def test_reservations_without_tokens(pg, ctx, D, N, groups):
    """Scans take what channels and states need, however many tokens; their gradient does not."""
    gen = torch.Generator().manual_seed(D)
    n, nseq = 3000, 4
    small = pg.Context(1000, 16, 5, 8, max_batch=1)
    small.reserve_selective(0, D, N)
    c = {k: cuda(v) for k, v in scan_inputs(gen, n, D, N, groups, nseq, "bf16").items()}
    o = torch.from_numpy(cuts(np.random.default_rng(D), n, nseq)).cuda()
    ins = (c["x"], c["delta"], c["A"], c["B"], c["C"])
    form = dict(state=c["h0"], skip=c["skip"], z=c["z"], delta_bias=c["bias"])
    want = ctx.selective_scan(*ins, o, marks=True, **form)
    for a, b in zip(small.selective_scan(*ins, o, marks=True, **form), want):
        assert torch.equal(a, b)
    with pytest.raises(pg.PolyglotError) as e:
        small.selective_backward(*ins, c["dy"], want[2], o, dlast=c["dlast"], **form)
    assert e.value.rc == pg.EBATCH
    w = normal(gen, D, 4).cuda()
    a, b = (k.convolution_backward(c["x"], w, None, c["dy"], o) for k in (small, ctx))
    assert torch.equal(a.x, b.x) and torch.equal(a.weight, b.weight)
    assert small.status() == pg.OK
    small.close()


def test_calls_without_last_states(pg, ctx):
    """last=False: no last states, and nothing of their size is allocated or written."""
    gen = torch.Generator().manual_seed(31)
    n, D, N, nseq = 600, 40, 16, 500
    c = {k: cuda(v) for k, v in scan_inputs(gen, n, D, N, 1, nseq, "f32").items()}
    o = torch.from_numpy(cuts(np.random.default_rng(31), n, nseq)).cuda()
    ins = (c["x"], c["delta"], c["A"], c["B"], c["C"])
    w = normal(gen, D, 4).cuda()
    for call, a in ((ctx.selective_scan, ins), (ctx.convolution, (c["x"], w, None))):
        want, last = call(*a, o)[:2]
        assert last is not None
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got = call(*a, o, last=False)
        assert torch.cuda.max_memory_allocated() - before < 2 * c["x"].nbytes
        assert got[1] is None and torch.equal(got[0], want)
    y, new = ctx.selective_step(*(t[:nseq] if t is not c["A"] else t for t in ins), c["h0"], last=False)
    assert new is None and torch.isfinite(y).all()
    y, new = ctx.convolution_step(c["x"][:nseq], w, None, last=False)
    assert new is None and torch.isfinite(y).all()
    for bad in (True, 0):
        with pytest.raises(TypeError):
            ctx.selective_scan(*ins, o, last=bad)


# ------------------------------------------------------------------ forms that sizes choose


def with_floor(err, tokens):
    """The references' bounds are relative.  A decay or a product below the least normal number,
    2^-126, may be off by as much as itself: at each token by 2^-126 times a state's size, and
    all of them leave by further factors (C, x, a step, A, sums over states and channels).
    States and their gradients stay below 2^10 in these tests, the factors together below 2^20."""
    return {k: v + tokens * 2.0 ** (-126 + 30) for k, v in err.items()}


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("tokens,D,N,groups,nseq", [(100, 130, 17, 1, 7), (333, 64, 32, 4, 30), (90, 70, 24, 2, 4),
                                                    (700, 33, 32, 1, 1), (1000, 9, 27, 3, 5)])
def test_selective_of_17_to_32_states(ctx, dtype, tokens, D, N, groups, nseq):
    rng = np.random.default_rng([tokens, D, N])
    off = cuts(rng, tokens, nseq)
    for form in range(3):
        gen = torch.Generator().manual_seed(tokens + D + form)
        s = scan_inputs(gen, tokens, D, N, groups, nseq, dtype, state=form != 1, gated=form != 2,
                        skip=form != 1, bias=form != 2)
        soft = form != 1
        if not soft:  # the step itself: not below zero
            s["delta"] = s["delta"].abs() * 0.25
            s["bias"] = s["bias"].abs() * 0.1
        o = torch.from_numpy(off).to(torch.int64 if form == 2 else torch.int32).cuda()
        want, err = scan_reference(s, off, soft, tokens)
        assert max(want[k].abs().max() for k in ("last", "state")) < 2 ** 10
        check_scan(scan_call(ctx, s, o, soft), want, with_floor(err, tokens), dtype, form)


def uneven(kind, tokens):
    """Offsets of one sequence, or of a long one among short and empty ones."""
    short = [3, 0, 7, 1, 0, 16, 17, 2] * 4
    long = tokens - sum(short)
    sizes = {"one": [tokens], "first": [long] + short, "last": short + [long],
             "middle": short[:16] + [long] + short[16:], "two": short + [long // 2] + short + [long - long // 2 - sum(short)]}
    off = np.concatenate([[0], np.cumsum(sizes[kind])]).astype(np.int64)
    assert off[-1] == tokens
    return off


@pytest.mark.parametrize("tokens,D,N,groups,kind", [
    (9000, 40, 32, 1, "first"), (9000, 40, 16, 1, "last"), (9000, 24, 4, 1, "middle"), (9001, 16, 40, 2, "two"),
    (12_000, 36, 24, 1, "one"), (20_005, 5, 4, 1, "one"), (20_005, 5, 16, 1, "middle"), (33_000, 3, 2, 1, "first"),
    (5000, 300, 8, 2, "two"), (3001, 1030, 4, 1, "last"), (2000, 24, 16, 1, "middle"), (1990, 40, 24, 1, "last")])
def test_selective_of_uneven_sequences(ctx, tokens, D, N, groups, kind):
    """A sequence through hundreds of ranges (and groups of them), alone and beside short ones.
    Values, and the same bits in two runs."""
    gen = torch.Generator().manual_seed(tokens + N)
    off = uneven(kind, tokens)
    s = scan_inputs(gen, tokens, D, N, groups, len(off) - 1, "f32")
    s["A"] = -torch.exp(normal(gen, D, N) - 1)
    s["bias"] = normal(gen, D) - 4
    o = torch.from_numpy(off).cuda()
    want, err = scan_reference(s, off, True, tokens)
    a = scan_call(ctx, s, o, True)
    check_scan(a, want, with_floor(err, tokens), "f32", kind)
    b = scan_call(ctx, s, o, True)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_replays_with_other_offsets(pg):
    """A captured scan and its gradient, replayed with sequences of other lengths: even ones, a
    long one first, in the middle and last, one alone beside empty ones."""
    stream = torch.cuda.Stream()
    gen = torch.Generator().manual_seed(41)
    n, D, N, nseq = 9000, 24, 16, 33
    c = {k: cuda(v) for k, v in scan_inputs(gen, n, D, N, 1, nseq, "f32").items()}
    c["bias"] -= 3
    even = np.linspace(0, n, nseq + 1).astype(np.int64)
    alone = np.concatenate([[0] * 5, [n] * (nseq - 4)])
    o = torch.from_numpy(even).cuda()
    with torch.cuda.stream(stream):
        ctx = pg.Context(1000, 16, 5, 8, max_batch=1, stream=stream)
        ctx.reserve_selective(n, D, N)

        def work():
            form = dict(state=c["h0"], skip=c["skip"], z=c["z"], delta_bias=c["bias"])
            ins = (c["x"], c["delta"], c["A"], c["B"], c["C"])
            y, last, marks = ctx.selective_scan(*ins, o, marks=True, **form)
            return [y, last, *ctx.selective_backward(*ins, c["dy"], marks, o, dlast=c["dlast"], **form)]

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = work()
        seen = []
        for off in (uneven("first", n), even, uneven("middle", n), alone, uneven("last", n), even):
            o.copy_(torch.from_numpy(off))
            graph.replay()
            torch.cuda.synchronize()
            first = [t.clone() for t in held]
            for a, e in zip(first, work()):
                assert torch.equal(a, e)
            torch.cuda.synchronize()
            seen.append(first[0])
        assert torch.equal(seen[1], seen[5]) and not torch.equal(seen[0], seen[1])
        assert ctx.status() == pg.OK
        ctx.close()


@pytest.mark.parametrize("bad", [[0, 5000, 3000, 9000], [0, 9000, 2_000_000_000, 9000], [8999, 0, 0, 0], [0, 0, 0, 0],
                                 [9000, 9000, 9000, 9000]])
def test_offsets_that_do_not_ascend_over_many_ranges(pg, ctx, bad):
    """The flag, and a right answer to the next call."""
    gen = torch.Generator().manual_seed(42)
    n, D, N = 9000, 24, 8
    s = scan_inputs(gen, n, D, N, 1, 3, "f32")
    good = torch.tensor([0, 10, 8990, n], dtype=torch.int32, device="cuda")
    want = scan_call(ctx, s, good, True)
    assert ctx.status() == pg.OK
    scan_call(ctx, s, torch.tensor(bad, dtype=torch.int32, device="cuda"), True)
    assert ctx.status() == pg.EOFFSETS and ctx.status() == pg.OK
    got = scan_call(ctx, s, good, True)
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("tokens,D,N,groups,nseq", [(9000, 40, 4, 1, 600), (9001, 36, 16, 2, 500), (6000, 20, 24, 1, 400),
                                                    (5000, 24, 64, 1, 300), (5003, 64, 4, 64, 3), (3001, 120, 32, 120, 1),
                                                    (9000, 40, 16, 1, 1), (2500, 300, 24, 1, 2)])
def test_selective_sums_that_are_exact(ctx, dtype, tokens, D, N, groups, nseq):
    """Whole numbers, decays of 1: every product and sum is a whole number below 2^24, so that
    32 bits hold it in any order, and a token that is lost or taken twice shows."""
    gen = torch.Generator().manual_seed(tokens + D)
    off = cuts(np.random.default_rng([tokens, D]), tokens, nseq)
    mean = tokens / nseq
    s = scan_inputs(gen, tokens, D, N, groups, nseq, dtype, gated=False)
    few = lambda *shape: torch.randint(-1, 2, shape, generator=gen).float()
    # what comes into a state, and back into it, is mostly zero where the sequence is long
    some = (torch.rand(tokens, 1, generator=gen) < min(1.0, 8 / mean)).float()
    s["x"] = few(tokens, D).to(DT[dtype])
    s["B"] = (some * few(tokens, groups * N)).to(DT[dtype])
    s["C"] = (some.flip(0) * few(tokens, groups * N)).to(DT[dtype])
    s["delta"] = torch.randint(1, 3, (tokens, D), generator=gen).float().to(DT[dtype])
    s["bias"], s["skip"], s["A"] = torch.zeros(D), few(D), torch.zeros(D, N)
    s["h0"], s["dlast"] = few(nseq, D, N), few(nseq, D, N)
    s["dy"] = few(tokens, D).to(DT[dtype])
    o = torch.from_numpy(off).cuda()
    want, _ = scan_reference(s, off, False, 0)
    got = scan_call(ctx, s, o, False)
    for k, v in want.items():
        assert v.abs().max() < 2 ** 24, k
        assert torch.equal(v, v.round()), k
    for k, v in got.items():
        if k in F32_OUT:
            assert torch.equal(wide(v), want[k]), (k, (wide(v) - want[k]).abs().max())
        else:
            assert torch.equal(v.cpu(), want[k].to(DT[dtype])), k


@pytest.mark.parametrize("kind", ["one", "first", "last"])
@pytest.mark.parametrize("tokens", [140_000, 280_000])
def test_selective_through_the_most_ranges(pg, tokens, kind):
    """A sequence through 1,000 and 2,000 ranges, whole numbers and decays of 1 as above; the
    states are running sums."""
    D, N = 3, 2
    ctx = pg.Context(1000, 16, 5, 8, max_batch=1)
    ctx.reserve_selective(tokens, D, N)
    gen = torch.Generator().manual_seed(tokens)
    off = uneven(kind, tokens)
    nseq = len(off) - 1
    few = lambda *shape: torch.randint(-1, 2, shape, generator=gen).float()
    some = lambda: (torch.rand(tokens, 1, generator=gen) < 40 / tokens).float()
    s = {"x": few(tokens, D), "delta": torch.randint(1, 3, (tokens, D), generator=gen).float(), "A": torch.zeros(D, N),
         "B": some() * few(tokens, N), "C": some() * few(tokens, N), "z": None, "skip": few(D), "bias": None,
         "h0": few(nseq, D, N), "dlast": few(nseq, D, N), "dy": few(tokens, D)}
    got = scan_call(ctx, s, torch.from_numpy(off).cuda(), False)
    w = {k: wide(v) for k, v in s.items()}
    u = (w["delta"] * w["x"]).unsqueeze(2) * w["B"].unsqueeze(1)
    into = w["dy"].unsqueeze(2) * w["C"].unsqueeze(1)
    h, before, lam = torch.empty_like(u), torch.empty_like(u), torch.empty_like(u)
    last, dh0 = torch.empty(nseq, D, N, dtype=torch.float64), torch.empty(nseq, D, N, dtype=torch.float64)
    for i, (a, z) in enumerate(zip(off, off[1:])):
        run = torch.cat([w["h0"][i][None], u[a:z]]).cumsum(0)
        h[a:z], before[a:z], last[i] = run[1:], run[:-1], run[-1]
        run = torch.cat([w["dlast"][i][None], into[a:z].flip(0)]).cumsum(0)
        lam[a:z], dh0[i] = run[1:].flip(0), run[-1]
    e = (lam * w["B"].unsqueeze(1)).sum(2)
    q = lam * before
    ddelta = w["x"] * e
    want = {"y": (h * w["C"].unsqueeze(1)).sum(2) + w["skip"] * w["x"], "last": last, "state": dh0,
            "x": w["delta"] * e + w["skip"] * w["dy"], "delta": ddelta, "A": (q * w["delta"].unsqueeze(2)).sum(0),
            "B": (lam * (w["delta"] * w["x"]).unsqueeze(2)).sum(1), "C": (w["dy"].unsqueeze(2) * h).sum(1),
            "skip": (w["dy"] * w["x"]).sum(0)}
    assert (q * w["delta"].unsqueeze(2)).abs().sum(0).max() < 2 ** 24
    for k, v in want.items():
        assert torch.equal(wide(got[k]), v), (k, (wide(got[k]) - v).abs().max())
    assert ctx.status() == pg.OK
    ctx.close()


# tokens, D, nseq, K: chunks of several steps of eight tokens, forward and back
LONG_CONV = [(40_000, 515, 3000, 4), (40_003, 515, 5, 4), (150_001, 130, 1500, 3), (300, 90_001, 40, 4),
             (77, 270_000, 9, 2), (700_001, 24, 3000, 4)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("tokens,D,nseq,K", LONG_CONV)
def test_convolution_of_long_chunks(ctx, dtype, tokens, D, nseq, K):
    """Against the formulas in a part of the channels, in every channel against calls of few
    channels, whose chunks are short, and the sums over tokens exactly."""
    if D > 1100:
        ctx.reserve_selective(0, D, 1)
    gen = torch.Generator(device="cuda").manual_seed(tokens + D)
    g = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    off = cuts(np.random.default_rng([tokens, D]), tokens, nseq)
    o = torch.from_numpy(off).to(torch.int32).cuda()
    x, dy = g(tokens, D).to(DT[dtype]), g(tokens, D).to(DT[dtype])
    w, b = g(D, K), g(D)
    st, dl = g(nseq, K - 1, D).to(DT[dtype]), g(nseq, K - 1, D).to(DT[dtype])
    y, last = ctx.convolution(x, w, b, o, state=st)
    d = ctx.convolution_backward(x, w, b, dy, o, state=st, dlast=dl)
    # some channels, the first and the last strips among them
    some = sorted({0, 1, 2, 3, 4, 7, 8, D // 2, *range(D - 10, D), min(D - 1, 255), min(D - 1, 256)})
    at = torch.tensor(some, device="cuda")
    part = lambda t: wide(t[..., at].contiguous())
    want, want_last, err = ref.conv(part(x), wide(w[at]), wide(b[at]), off, part(st), True)
    near(y[:, at], want, ref.rounded(err, want, dtype), "y")
    assert torch.equal(part(last), want_last)
    want, errs = ref.conv_grad(part(x), wide(w[at]), wide(b[at]), part(dy), off, part(st), part(dl), True)
    near(d.x[:, at], want[0], ref.rounded(errs[0], want[0], dtype), "dx")
    near(d.weight[at], want[1], ref.rounded(errs[1], want[1], "f32"), "dw")
    near(d.bias[at], want[2], ref.rounded(errs[2], want[2], "f32"), "db")
    near(d.state[..., at], want[3], ref.rounded(errs[3], want[3], dtype), "dstate")
    # the first tokens of all channels, in a call whose rows are short chunks
    n = min(tokens, 512 if D < 2000 else 24)
    s = int(np.searchsorted(off, n, side="right")) - 1  # the whole sequences within them
    if s > 0:
        n = int(off[s])
        head = lambda t: t[:s].contiguous()
        for lo in range(0, D, 4096):
            c = slice(lo, min(D, lo + 4096))
            short = ctx.convolution(x[:n, c], w[c], b[c], o[:s + 1], state=head(st[..., c]))
            assert torch.equal(short[0], y[:n, c]) and torch.equal(short[1], last[:s, :, c]), lo
            back = ctx.convolution_backward(x[:n, c], w[c], b[c], dy[:n, c], o[:s + 1], state=head(st[..., c]),
                                            dlast=head(dl[..., c]))
            assert torch.equal(back.x, d.x[:n, c]) and torch.equal(back.state, d.state[:s, :, c]), lo
    # whole numbers without silu: sums below 2^24, exact in any order
    ints = lambda *shape: torch.randint(-2, 3, shape, generator=gen, device="cuda").to(DT[dtype])
    x, dy, w = ints(tokens, D), ints(tokens, D), ints(D, K).float()
    d = ctx.convolution_backward(x, w, b, dy, o, silu=False)
    seq = torch.from_numpy(np.repeat(off[:-1], np.diff(off))).cuda()  # where each token's sequence starts
    t = torch.arange(tokens, device="cuda")
    for k in range(K):
        back = K - 1 - k
        inside = (t - back >= seq).unsqueeze(1)
        taken = torch.where(inside, x[(t - back).clamp(min=0)], torch.zeros((), dtype=x.dtype, device="cuda"))
        total = torch.cat([(taken[:, i:i + 20_000].float() * dy[:, i:i + 20_000].float()).sum(0, dtype=torch.float64)
                           for i in range(0, D, 20_000)])
        assert torch.equal(d.weight[:, k].double(), total), k
    assert torch.equal(d.bias.double(), dy.float().sum(0, dtype=torch.float64))
    if D > 1100:
        ctx.reserve_selective(70_000, 1100, 64)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("groups,beams,V,picks", [(32, 8, 32_003, 16), (16, 8, 32_003, 64), (64, 8, 8193, 64),
                                                  (33, 4, 40_000, 5), (2, 256, 16_385, 3)])
def test_beams_of_long_parts(ctx, dtype, groups, beams, V, picks):
    """Parts of 8,192 and 16,384 words: ordinary scores, and few values that tie everywhere."""
    gen = torch.Generator().manual_seed(V + beams)
    rows = groups * beams
    total, lse = normal(gen, rows) - 20, normal(gen, rows) + 8
    over = (torch.rand(rows, generator=gen) < 0.3).to(torch.int32)
    for kind in ("scores", "ties"):
        if kind == "scores":
            scores = normal(gen, rows, V, dtype=dtype, std=2.0)
            scores[0, 5], scores[0, 17] = math.nan, -math.inf
        else:
            scores = torch.randint(0, 3, (rows, V), generator=gen).to(DT[dtype])
            total, lse = torch.zeros(rows), torch.ones(rows)
        want = ref.beam(scores.float().numpy(), total.numpy(), lse.numpy(), beams, picks, over.numpy(), 1)
        got = ctx.beam(cuda(scores), cuda(total), beams=beams, picks=picks, lse=cuda(lse), finished=cuda(over), end=1)
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w), kind
