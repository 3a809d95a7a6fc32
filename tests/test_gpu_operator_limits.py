"""The sequence operators at the limits of what a launch, a tag or a format holds, and
the variants of their kernels that sizes choose."""
import pytest

from test_gpu_operators import Scores, Seqs, ctx, dev, host, near, pg  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_scores_of_more_rows_than_a_launch_has(pg):  # noqa: F811
    """2^24 workgroups are more than a launch takes: every row against a call of fewer rows."""
    rows, V = 2 ** 24 + 5, 3
    c = pg.Context(1000, 16, 5, 8, max_batch=1)
    c.reserve_logits(rows, V)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    ints = lambda lo, hi, *s: torch.randint(  # noqa: E731
        lo, hi, s, device="cuda", generator=gen, dtype=torch.int32)
    x = rand(rows, V).half()
    kw = dict(history=ints(-1, V, rows, 2), lengths=ints(0, 3, rows), prompt=ints(0, 3, rows),
              repetition=rand(rows).abs() + 0.5, presence=rand(rows), frequency=rand(rows),
              bias=rand(rows, V), mask=ints(0, 8, rows, 1))
    got = c.logits(x, **kw)
    for a, b in ((0, 2 ** 23), (2 ** 23, 2 ** 24 - 100), (2 ** 24 - 100, rows)):
        want = c.logits(x[a:b], **{k: v[a:b] for k, v in kw.items()})
        for g, w in zip(got, want):
            assert torch.equal(g[a:b], w), (a, b)
    assert c.status() == pg.OK
    c.close()


def set_stream(pg, c, stream):  # noqa: F811
    assert pg.load_library().polyglot_set_stream(c._h, stream.cuda_stream) == pg.OK


def test_calls_after_a_change_of_the_stream_wait(pg):  # noqa: F811
    """Two streams in turn, nothing waited for in between: the scans share the tickets and
    the rows of scores their counters."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.default_stream()]
    c = pg.Context(1000, 16, 5, 8, max_batch=1, stream=streams[0])
    c.reserve_recurrence(20_000, 512)
    c.reserve_logits(8, 100_000)
    gen = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    sets = [(rand(20_000, 512), rand(20_000, 512), rand(8, 100_000)) for _ in range(3)]
    outs = [(torch.empty_like(g), torch.empty(1, 512, device="cuda")) for g, _, _ in sets]
    torch.cuda.synchronize()

    def run(k):
        gate, x, scores = sets[k]
        with torch.cuda.stream(streams[k]):
            c.recurrence(gate, x, out=outs[k][0], last=outs[k][1])
            return c.logits(scores)

    want = []
    for k in range(3):
        set_stream(pg, c, streams[k])
        got = run(k)
        torch.cuda.synchronize()
        want.append([t.clone() for t in (*outs[k], *got)])
    for _ in range(20):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        got = []
        for k in range(3):
            set_stream(pg, c, streams[k])
            got.append(run(k))
        torch.cuda.synchronize()
        for k in range(3):
            assert all(torch.equal(a, b) for a, b in zip((*outs[k], *got[k]), want[k])), k
    assert c.status() == pg.OK
    c.close()


def test_a_change_of_the_stream_into_a_capture(pg):  # noqa: F811
    """A context that works eagerly lends its calls to a capture and takes them back."""
    c = pg.Context(1000, 16, 5, 8, max_batch=1, stream=torch.cuda.default_stream())
    c.reserve_recurrence(4000, 64)
    q = Seqs("f32", [1500, 0, 900], 64, 1, True, seed=31)
    off, h, last = q.offsets(), torch.empty_like(q.x), torch.empty_like(q.h0)
    call = lambda: c.recurrence(q.gate, q.x, off, h0=q.h0, out=h, last=last)  # noqa: E731
    call()
    torch.cuda.synchronize()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        set_stream(pg, c, s)
        call()
        set_stream(pg, c, torch.cuda.default_stream())
    for k in range(4):
        call()
        torch.cuda.synchronize()
        want = h.clone(), last.clone()
        h.zero_()
        last.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, want[0]) and torch.equal(last, want[1]), k
        q.x.mul_(1.25)
        torch.cuda.synchronize()
    assert c.status() == pg.OK
    c.close()
