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
