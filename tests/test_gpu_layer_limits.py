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
