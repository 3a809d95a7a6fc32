"""The example model that uses the sequence operators together: it learns, it
answers within its grammar, and its training step's gradient is autograd's."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lm():
    spec = importlib.util.spec_from_file_location("recurrent_lm",
                                                  os.path.join(ROOT, "examples", "recurrent_lm.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_learns_and_answers(lm):
    losses, named, held, logp = lm.main(steps=300, quiet=True)
    assert np.isfinite(losses).all()
    assert abs(losses[0] - 1) < 0.2  # untrained scores differ by little: the margin of one
    assert np.mean(losses[-50:]) < 0.35  # one word in ten follows no rule
    assert named > 0.6  # and the rule's word is the best of 200 most of the time
    assert (held[:, 1:] % 2 != held[:, :-1] % 2).all()  # odd after even, even after odd
    assert all(len(set(row)) == len(row) for row in held.tolist())  # nothing twice
    assert (logp <= 1e-5).all()


def test_training_step_against_autograd(lm):
    """The step's updates of all parameters against autograd in 64 bits, the recurrence
    written out token by token, with the mask that the dropout computed."""
    corpus = lm.Corpus(60, seed=3)
    m = lm.Model(60, 24, max_tokens=400, max_live=4, seed=5)
    words, follows, offsets = corpus.batch(9)
    random = torch.from_numpy(np.random.default_rng(4).integers(0, 60, words.shape[0])
                              .astype(np.int32)).cuda()
    old = {k: getattr(m, k).double().cpu().requires_grad_() for k in ("E", "O", "Wg", "Wx", "bg")}
    kept = m.ctx.dropout(torch.ones(words.shape[0], 24, device="cuda"), 0.25, 5, site=7).double().cpu()
    lr = 0.5
    loss = m.train_step(words, follows, offsets, random, lr, 0.25, 7)

    w, f, r = (t.cpu().long() for t in (words, follows, random))
    e = old["E"][w] * kept
    a, x = torch.sigmoid(e @ old["Wg"].T + old["bg"]), e @ old["Wx"].T
    rows, off = [], offsets.tolist()
    for s in range(len(off) - 1):
        h = torch.zeros(24, dtype=torch.float64)
        for t in range(off[s], off[s + 1]):
            h = a[t] * h + (1 - a[t]) * x[t]
            rows.append(h)
    h = torch.stack(rows)
    ref = (1 - (h * (old["O"][f] - old["O"][r])).sum(1)).clamp(min=0).mean()
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) < 1e-5
    for k, p in old.items():
        got = (p.detach() - getattr(m, k).double().cpu()) / lr
        # float32 throughout: roundings of some hundred products and sums, and of the
        # parameter itself, half a unit of which the division by lr brings up
        size = float(p.grad.abs().max())
        tol = 2e-5 * size + 2.0 ** -24 * float(p.abs().max()) / lr * 2
        assert float((got - p.grad).abs().max()) <= tol, k
    assert m.ctx.status() == 0
