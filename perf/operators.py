"""Cases of the sequence operators: dropout without a stored mask, the gated
linear recurrence over packed sequences, and the penalties, biases and grammar
masks on the scores of a vocabulary.

The three are the parts of a recurrent language model on the framework's word
table.  Training: rows gathered with dropout, the recurrence, its gradient, the
dropout's gradient.  Answering: one token for every live sequence, then the
choice among the vocabulary's scores.

A case is a dict of plain values; ``kind`` says what is called:

  dropout     Context.dropout, rows of an input or of a table by their ids
  dropgrad    Context.dropout and Context.dropout_backward: a training step's two
  step        Context.recurrence_step: one token for every live sequence
  forward     Context.recurrence
  backward    Context.recurrence_backward
  logits      Context.logits

The plain forms below are elementary torch operations in 32 bits.  Widths and
vocabularies are those of the workload presets (64, 128 and 256 wide, 100,000
and 1,000,000 words) and of wider layers.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GATE = {"raw": 0, "sigmoid": 1}  # POLYGLOT_GATE_*


def _drop(name, kind, dtype, rows, d, p, table=0, residual=False, whole=False):
    return {"name": name, "kind": kind, "dtype": dtype, "rows": rows, "d": d, "p": p,
            "table": table, "residual": residual, "whole": whole}


def _rec(name, kind, dtype, tokens, D, nseq, group=1, form="sigmoid", reverse=False, state=False):
    return {"name": name, "kind": kind, "dtype": dtype, "tokens": tokens, "D": D, "nseq": nseq,
            "group": group, "form": form, "reverse": reverse, "state": state}


def _log(name, dtype, rows, V, hist, masks, bias):
    return {"name": name, "kind": "logits", "dtype": dtype, "rows": rows, "V": V, "hist": hist,
            "masks": masks, "bias": bias}


def listed():
    return [
        # the words of a minibatch of 1,024 windows of five, gathered with dropout
        _drop("drop-words-5120", "dropout", "f32", 5120, 64, 0.1, table=100_000),
        # a layer's output of an odd width dropped and added to its input
        _drop("drop-add-20011x199", "dropout", "bf16", 20_011, 199, 0.25, residual=True),
        # a large step's activations: dropout going in, its gradient coming back
        _drop("drop-step-262144x512", "dropgrad", "f16", 262_144, 512, 0.1),
        # 64 live sequences, the next word of each: what latency costs
        _rec("step-64x256", "step", "bf16", 64, 256, 64, state=True),
        # a minibatch of sentences, in the table's own width and type
        _rec("fwd-sentences-128", "forward", "f32", 16_384, 128, 700),
        # the gradient of sentences of all lengths, one gate for 32 channels
        _rec("bwd-sentences-256", "backward", "bf16", 16_411, 256, 700, group=32),
        # one book in a single sequence, from right to left, gates as they are
        _rec("bwd-book-64", "backward", "f32", 65_537, 64, 1, form="raw", reverse=True, state=True),
        # 16 documents through a wide layer
        _rec("fwd-documents-2048", "forward", "bf16", 65_536, 2048, 16, state=True),
        # ... and the gradient of that layer
        _rec("bwd-documents-2048", "backward", "bf16", 65_536, 2048, 16, state=True),
        # one live sequence over the presets' vocabulary
        _log("scores-1x100000", "f32", 1, 100_000, 200, 1, True),
        # a serving batch, a vocabulary that no word width divides, a grammar state for each
        _log("scores-48x32003", "bf16", 48, 32_003, 1024, 12, True),
        # a large batch over the largest vocabulary
        _log("scores-256x1000000", "bf16", 256, 1_000_000, 4096, 4, False),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["dropout", "dropgrad", "step", "forward", "forward", "backward", "backward",
                       "logits", "logits"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind in ("dropout", "dropgrad"):
        d = _spread(rng, 16, 4096)
        rows = _spread(rng, 8, max(64, min(1_000_000, 60_000_000 // d)))
        table = 0
        if kind == "dropout" and rng.random() < 0.4:
            d = rng.choice([16, 64, 100, 128, 256])
            rows = _spread(rng, 100, 300_000)
            table = _spread(rng, 1000, 300_000)
        c = _drop("", kind, dtype, rows, d, rng.choice([0.05, 0.1, 0.25, 0.5]), table=table,
                  residual=kind == "dropout" and rng.random() < 0.5, whole=rng.random() < 0.2)
    elif kind == "step":
        D = _spread(rng, 16, 4096)
        n = _spread(rng, 1, 2048)
        c = _rec("", kind, dtype, n, D, n, group=rng.choice([1, 1, 16, D if D <= 256 else 1]),
                 form=rng.choice(["sigmoid", "raw"]), state=True)
    elif kind in ("forward", "backward"):
        D = _spread(rng, 16, 2048)
        tokens = _spread(rng, 64, min(100_000, 60_000_000 // D))
        nseq = _spread(rng, 1, max(2, tokens // 8))
        c = _rec("", kind, dtype, tokens, D, nseq, group=rng.choice([1, 1, 16, 32, 64]),
                 form=rng.choice(["sigmoid", "raw"]), reverse=rng.random() < 0.5,
                 state=rng.random() < 0.5)
    else:
        V = _spread(rng, 1000, 1_000_000)
        rows = _spread(rng, 1, max(2, min(512, 60_000_000 // V)))
        c = _log("", dtype, rows, V, _spread(rng, 16, 4096), rng.choice([0, 1, rows]),
                 rng.random() < 0.5)
    if "group" in c:  # a width that the heads divide
        c["D"] = max(1, c["D"] // c["group"]) * c["group"]
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    x = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=gen)
    return x.to(dtype)


def _zipf(gen, shape, V):
    """Word ids of a frequency-ranked vocabulary: the rank is log-uniform."""
    u = torch.rand(shape, device="cuda", generator=gen, dtype=torch.float64)
    return (torch.exp(u * math.log(V)) - 1).to(torch.int32).clamp_(0, V - 1)


def _cuts(rng, tokens, nseq):
    """Offsets of nseq sequences of all lengths, a few of them empty."""
    cut = np.sort(rng.integers(0, tokens + 1, nseq - 1))
    return np.concatenate([[0], cut, [tokens]]).astype(np.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = DTYPES[case["dtype"]]
    s = dict(case)
    if case["kind"] in ("dropout", "dropgrad"):
        rows, d = case["rows"], case["d"]
        s["seed"] = int(rng.integers(0, 1 << 62))
        s["site"] = int(rng.integers(0, 1000))
        s["x"] = _normal(gen, (case["table"] or rows, d), dt)
        s["ids"] = _zipf(gen, (rows,), case["table"]) if case["table"] else None
        s["add"] = _normal(gen, (rows, d), dt) if case["residual"] else None
        s["dy"] = _normal(gen, (rows, d), dt) if case["kind"] == "dropgrad" else None
    elif case["kind"] == "logits":
        rows, V, cap = case["rows"], case["V"], case["hist"]
        s["logits"] = _normal(gen, (rows, V), dt, 3.0)
        s["history"] = _zipf(gen, (rows, cap), V)
        length = torch.randint(0, cap + 1, (rows,), device="cuda", generator=gen)
        s["lengths"] = length.to(torch.int32)
        part = torch.rand(rows, device="cuda", generator=gen)
        s["prompt"] = (length * part).to(torch.int32)
        u = torch.rand(3, rows, device="cuda", generator=gen)
        s["repetition"] = 1.0 + 0.3 * u[0]
        s["presence"] = 0.5 * u[1]
        s["frequency"] = 0.2 * u[2]
        s["bias"] = _normal(gen, (V,), torch.float32, 0.5) if case["bias"] else None
        s["mask"] = s["mask_rows"] = None
        if case["masks"]:
            words = (V + 31) // 32
            bits = torch.randint(0, 1 << 32, (2, case["masks"], words), device="cuda",
                                 generator=gen, dtype=torch.int64)
            # a grammar state allows every word, half of them or a quarter
            share = torch.randint(0, 3, (case["masks"], 1), device="cuda", generator=gen)
            w = torch.where(share == 0, 0xFFFFFFFF, torch.where(share == 1, bits[0],
                                                                bits[0] & bits[1]))
            s["mask"] = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
            s["mask_rows"] = torch.randint(-1, case["masks"], (rows,), device="cuda",
                                           generator=gen).to(torch.int32)
    else:
        n, D, nseq = case["tokens"], case["D"], case["nseq"]
        gates = D // case["group"] if case["group"] > 1 else D
        if case["form"] == "raw":  # decays of a few to a few hundred tokens
            u = torch.rand(n, gates, device="cuda", generator=gen)
            s["gate"] = (1.0 - torch.exp(-1.0 - 4.0 * u)).to(dt)
        else:
            s["gate"] = _normal(gen, (n, gates), dt, 1.5, 2.0)
        s["x"] = _normal(gen, (n, D), dt)
        s["h0"] = _normal(gen, (nseq, D), torch.float32) if case["state"] else None
        if case["kind"] != "step":
            off = _cuts(rng, n, nseq)
            s["longest"] = int(np.diff(off).max())
            s["offsets"] = torch.from_numpy(off).cuda()
        if case["kind"] == "backward":
            s["dh"] = _normal(gen, (n, D), dt)
            s["dlast"] = _normal(gen, (nseq, D), torch.float32) if case["state"] else None
            s["h"] = _plain_forward(s)[0]  # a training step has it from its forward pass
    return s


# ------------------------------------------------------------------ plain forms


def _plain_kept(seed, site, rows, d, p, whole):
    """Which elements of [rows][d] stay: the 16-bit pieces of Philox 4x32-10 (Salmon et
    al., SC 2011) at the counter (column / 8, row, site) and the key `seed`, each against
    round(65536 p).  Whole rows go by the first piece at column group 2^32 - 1."""
    M = 0xFFFFFFFF
    groups = 1 if whole else (d + 7) // 8
    r = torch.arange(rows, device="cuda").unsqueeze(1).expand(rows, groups)
    c0 = torch.full_like(r, M) if whole else torch.arange(groups, device="cuda").expand_as(r)
    c1, c2, c3 = r & M, r >> 32, torch.full_like(r, site)
    k0, k1 = seed & M, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # modulo 2^64: the low 64 bits are exact
        c0, c1, c2, c3 = ((p1 >> 32) & M) ^ c1 ^ k0, p1 & M, ((p0 >> 32) & M) ^ c3 ^ k1, p0 & M
        k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
    piece = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16,
                         c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 2)
    kept = piece >= int(p * 65536 + 0.5)
    return kept[:, 0, :1].expand(rows, d) if whole else kept.reshape(rows, groups * 8)[:, :d]


def _plain_dropout(x, kept, p, add=None):
    thr = int(p * 65536 + 0.5)
    y = torch.where(kept, x.float() * (65536.0 / (65536 - thr)), 0.0)
    return (y if add is None else y + add.float()).to(x.dtype)


def _plain_scan(a, b, longest):
    """h_t = a_t h_{t-1} + b_t down the rows, by doubling; a is 0 where a sequence starts."""
    step = 1
    while step < longest:
        b = torch.cat([b[:step], a[step:] * b[:-step] + b[step:]])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return b


def _plain_gates(s):
    """The decays and, for gates given before their sigmoid, one minus them."""
    g = s["gate"].float().repeat_interleave(s["group"], 1)
    if s["form"] == "raw":
        return g, None
    return 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))


def _plain_places(s):
    """Sequence of each token, and whether it is the first and the last that a pass meets."""
    off = s["offsets"].long()
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(off[1:].contiguous(), t, right=True)
    ends = (t == off[seq]).unsqueeze(1), (t == off[seq + 1] - 1).unsqueeze(1)
    return off, seq, *(ends[::-1] if s["reverse"] else ends)


def _plain_forward(s):
    off, seq, first, _ = _plain_places(s)
    a, rest = _plain_gates(s)
    x = s["x"].float()
    b = x if rest is None else rest * x
    start = s["h0"][seq] if s["h0"] is not None else torch.zeros_like(x)
    b = torch.where(first, a * start + b, b)
    a = torch.where(first, 0.0, a)
    if s["reverse"]:
        a, b = a.flip(0), b.flip(0)
    h = _plain_scan(a, b, s["longest"])
    if s["reverse"]:
        h = h.flip(0)
    at = off[:-1] if s["reverse"] else off[1:] - 1
    empty = (off[1:] == off[:-1]).unsqueeze(1)
    none = s["h0"] if s["h0"] is not None else 0.0
    last = torch.where(empty, none, h[at.clamp(0, s["tokens"] - 1)])
    return h.to(s["x"].dtype), last


def _plain_backward(s):
    off, seq, first, last = _plain_places(s)
    a, rest = _plain_gates(s)
    x, h, dh = s["x"].float(), s["h"].float(), s["dh"].float()
    zero = torch.zeros_like(x)
    start = s["h0"][seq] if s["h0"] is not None else zero
    end = s["dlast"][seq] if s["dlast"] is not None else zero
    back = 1 if s["reverse"] else -1  # where the token before is
    before = torch.where(first, start, h.roll(-back, 0))
    b = a * torch.where(last, dh + end, dh)
    decay = torch.where(last, 0.0, a)
    if not s["reverse"]:
        b, decay = b.flip(0), decay.flip(0)
    mu = _plain_scan(decay, b, s["longest"])
    if not s["reverse"]:
        mu = mu.flip(0)
    lam = dh + torch.where(last, end, mu.roll(back, 0))
    if rest is None:
        dx, dg = lam, lam * before
    else:
        dx, dg = rest * lam, a * rest * lam * (before - x)
    if s["group"] > 1:
        dg = dg.reshape(s["tokens"], -1, s["group"]).sum(2)
    if s["h0"] is None:
        return dg.to(s["x"].dtype), dx.to(s["x"].dtype), None
    at = off[1:] - 1 if s["reverse"] else off[:-1]
    empty = (off[1:] == off[:-1]).unsqueeze(1)
    none = s["dlast"] if s["dlast"] is not None else 0.0
    dh0 = torch.where(empty, none, mu[at.clamp(0, s["tokens"] - 1)])
    return dg.to(s["x"].dtype), dx.to(s["x"].dtype), dh0


def _plain_step(s):
    a, rest = _plain_gates(s)
    x = s["x"].float()
    h = a * s["h0"] + (x if rest is None else rest * x)
    return h.to(s["x"].dtype), h


def _plain_logits(s):
    rows, V = s["rows"], s["V"]
    l = s["logits"].float()
    k = torch.arange(s["hist"], device="cuda")
    live = k < s["lengths"].unsqueeze(1)
    made = live & (k >= s["prompt"].unsqueeze(1))
    ids = s["history"].long()
    seen = torch.zeros(rows, V, dtype=torch.int32, device="cuda")
    n = torch.zeros(rows, V, dtype=torch.int32, device="cuda")
    seen.scatter_add_(1, ids, live.int())
    n.scatter_add_(1, ids, made.int())
    rep, pres, freq = (s[w].unsqueeze(1) for w in ("repetition", "presence", "frequency"))
    l = torch.where(seen > 0, torch.where(l > 0, l / rep, l * rep), l)
    l = torch.where(n > 0, l - (freq * n + pres), l)
    if s["bias"] is not None:
        l = l + s["bias"]
    v = torch.arange(V, device="cuda")
    if s["mask"] is not None:
        words = s["mask"][s["mask_rows"].clamp(min=0).long()]
        allowed = ((words[:, v >> 5] >> (v & 31)) & 1) != 0
        allowed = allowed | (s["mask_rows"] < 0).unsqueeze(1)
        l = torch.where(allowed, l, -math.inf)
    best = l.amax(1, keepdim=True)
    token = torch.where(l == best, v, V).amin(1)
    token = torch.where(best[:, 0] == -math.inf, -1, token).to(torch.int32)
    base = torch.where(best == -math.inf, 0.0, best)
    lse = base[:, 0] + torch.log(torch.exp(l - base).sum(1))
    return l.to(s["logits"].dtype), token, lse


# ------------------------------------------------------------------ one pass

_CTX = None


def _context(tokens=0, width=0, rows=0, vocab=0):
    """The program's context.  Its workspace for the scan and for the join of a
    vocabulary's parts grows to the largest call that the program has made."""
    global _CTX
    import paper_1404_1521_amd as pg
    if _CTX is None:
        _CTX = (pg.Context(1000, 64, 5, 32, max_batch=32), [0, 0], [0, 0])
    ctx, rec, log = _CTX
    if tokens > rec[0] or width > rec[1]:
        rec[:] = max(tokens, rec[0]), max(width, rec[1])
        ctx.reserve_recurrence(*rec)
    if rows > log[0] or vocab > log[1]:
        log[:] = max(rows, log[0]), max(vocab, log[1])
        ctx.reserve_logits(*log)
    return ctx


def _own_run(s):
    kind = s["kind"]
    if kind in ("dropout", "dropgrad"):
        ctx = _context()
        y = ctx.dropout(s["x"], s["p"], s["seed"], site=s["site"], ids=s["ids"], add=s["add"],
                        whole_rows=s["whole"])
        if kind == "dropout":
            return y
        return y, ctx.dropout_backward(s["dy"], s["p"], s["seed"], site=s["site"],
                                       whole_rows=s["whole"])
    if kind == "logits":
        ctx = _context(rows=s["rows"], vocab=s["V"])
        return ctx.logits(s["logits"], history=s["history"], lengths=s["lengths"],
                          prompt=s["prompt"], repetition=s["repetition"], presence=s["presence"],
                          frequency=s["frequency"], bias=s["bias"], mask=s["mask"],
                          mask_rows=s["mask_rows"])
    form = GATE[s["form"]]
    if kind == "step":
        return _context().recurrence_step(s["gate"], s["x"], s["h0"], form=form)
    ctx = _context(s["tokens"], s["D"])
    if kind == "forward":
        return ctx.recurrence(s["gate"], s["x"], s["offsets"], h0=s["h0"], form=form,
                              reverse=s["reverse"])
    return ctx.recurrence_backward(s["gate"], s["x"], s["h"], s["dh"], s["offsets"], h0=s["h0"],
                                   dlast=s["dlast"], form=form, reverse=s["reverse"])


def run(s):
    if own:
        return _own_run(s)
    kind = s["kind"]
    if kind in ("dropout", "dropgrad"):
        kept = _plain_kept(s["seed"], s["site"], s["rows"], s["d"], s["p"], s["whole"])
        x = s["x"] if s["ids"] is None else s["x"][s["ids"].long()]
        y = _plain_dropout(x, kept, s["p"], s["add"])
        return y if kind == "dropout" else (y, _plain_dropout(s["dy"], kept, s["p"]))
    return {"logits": _plain_logits, "step": _plain_step, "forward": _plain_forward,
            "backward": _plain_backward}[kind](s)


def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] in ("dropout", "dropgrad"):
        n = case["rows"] * case["d"]
        read = n
        if case["table"]:  # the rows of the table that the ids reach, about: the ranks are log-uniform
            ln = math.log(case["table"])
            reach = case["rows"] / ln
            distinct = reach * (1 + math.log(case["table"] / reach)) if reach < case["table"] \
                else case["table"]
            read = min(case["rows"], distinct) * case["d"]
        b = (read + n + (n if case["residual"] else 0)) * e + (4 * case["rows"] if case["table"] else 0)
        m = 2 if case["kind"] == "dropgrad" else 1
        return {"bytes": m * b, "flops": m * n}
    if case["kind"] == "logits":
        n, rows = case["rows"] * case["V"], case["rows"]
        b = 2 * e * n + 4 * rows * (case["hist"] // 2 + 7) + (4 * case["V"] if case["bias"] else 0)
        return {"bytes": b + case["masks"] * case["V"] // 8, "flops": 4 * n}
    n, D = case["tokens"], case["D"]
    gates = D // case["group"]
    raw = case["form"] == "raw"
    per_seq = 4 * case["nseq"] * D
    if case["kind"] in ("step", "forward"):
        b = e * n * (gates + 2 * D) + per_seq * (2 if case["state"] else 1)
        return {"bytes": b, "flops": n * D * (2 if raw else 3) + n * gates * (0 if raw else 4)}
    b = e * n * (2 * gates + (3 if raw else 4) * D) + per_seq * (3 if case["state"] else 0)
    return {"bytes": b, "flops": n * D * (6 if raw else 8) + n * gates * (0 if raw else 6)}


# ------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    s = prepare(case, seed)

    def host(t):
        return None if t is None else t.double().cpu().numpy()

    if case["kind"] in ("dropout", "dropgrad"):
        rows, d, p = case["rows"], case["d"], case["p"]
        n8 = 1 if case["whole"] else -(-d // 8)

        def high_low(m, c):
            """The 64-bit product of two words below 2^32, from 16-bit halves."""
            low, mid = (c & 0xFFFF) * m, (c >> 16) * m
            total_low = low + ((mid & 0xFFFF) << 16)
            return (mid >> 16) + (total_low >> 32), total_low & 0xFFFFFFFF

        word = [torch.empty(rows, n8, dtype=torch.int64, device="cuda") for _ in range(4)]
        word[0][:] = 0xFFFFFFFF if case["whole"] else torch.arange(n8, device="cuda")
        word[1][:] = torch.arange(rows, device="cuda")[:, None]
        word[2][:] = 0
        word[3][:] = s["site"]
        key = [s["seed"] % (1 << 32), s["seed"] // (1 << 32)]
        for _ in range(10):
            h0, l0 = high_low(0xD2511F53, word[0])
            h1, l1 = high_low(0xCD9E8D57, word[2])
            word = [h1 ^ word[1] ^ key[0], l1, h0 ^ word[3] ^ key[1], l0]
            key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
        limit = int(p * 65536 + 0.5)
        kept = torch.empty(rows, n8, 8, dtype=torch.bool, device="cuda")
        for j in range(8):
            kept[:, :, j] = (word[j // 2] >> (16 * (j % 2))) % 65536 >= limit
        kept = kept[:, 0, :1].repeat(1, d) if case["whole"] else kept.view(rows, -1)[:, :d]
        x = s["x"] if s["ids"] is None else s["x"].index_select(0, s["ids"])
        y = x.double() * kept / (1 - limit / 65536)
        if s["add"] is not None:
            y += s["add"].double()
        return y if s["dy"] is None else (y, s["dy"].double() * kept / (1 - limit / 65536))

    if case["kind"] == "logits":
        rows, V = case["rows"], case["V"]
        outs, toks, lses = [], [], []
        for r in range(rows):
            l = s["logits"][r].double()
            ids = s["history"][r, : int(s["lengths"][r])].long()
            rep, pres, freq = (float(s[w][r]) for w in ("repetition", "presence", "frequency"))
            u = torch.unique(ids)
            l[u] = torch.where(l[u] > 0, l[u] / rep, l[u] * rep)
            u, c = torch.unique(ids[int(s["prompt"][r]):], return_counts=True)
            l[u] -= freq * c.double() + pres
            if s["bias"] is not None:
                l += s["bias"].double()
            if s["mask"] is not None and int(s["mask_rows"][r]) >= 0:
                w = s["mask"][int(s["mask_rows"][r])].long()
                bit = (w[:, None] >> torch.arange(32, device="cuda")[None]) % 2
                l[bit.view(-1)[:V] == 0] = -math.inf
            outs.append(l)
            lses.append(torch.logsumexp(l, 0))
        # the token goes by 32-bit comparisons of the 32-bit scores: no value of its own here
        return torch.stack(outs), None, torch.stack(lses)

    sig = case["form"] == "sigmoid"
    g = host(s["gate"])
    a = 1 / (1 + np.exp(-g)) if sig else g
    rest = 1 / (1 + np.exp(g)) if sig else np.ones_like(g)
    a, rest = np.repeat(a, case["group"], 1), np.repeat(rest, case["group"], 1)
    x, h0 = host(s["x"]), host(s["h0"])
    if case["kind"] == "step":
        h = a * h0 + rest * x
        return torch.from_numpy(h), torch.from_numpy(h)
    off = s["offsets"].cpu().numpy().astype(np.int64)
    nseq, D = case["nseq"], case["D"]
    size = np.diff(off)
    order = np.argsort(-size, kind="stable")  # the live sequences of a step come first
    live = np.searchsorted(-size[order], -np.arange(s["longest"]), side="left")
    up = 1 if not case["reverse"] else -1
    head = off[:-1] if up == 1 else off[1:] - 1  # a sequence's first token
    if case["kind"] == "forward":
        state = np.zeros((nseq, D)) if h0 is None else h0.copy()
        h = np.empty_like(x)
        for t in range(s["longest"]):
            q = order[: live[t]]
            k = head[q] + up * t
            state[q] = a[k] * state[q] + rest[k] * x[k]
            h[k] = state[q]
        return torch.from_numpy(h), torch.from_numpy(state)
    h, dh = host(s["h"]), host(s["dh"])
    mu = np.zeros((nseq, D)) if s["dlast"] is None else host(s["dlast"])
    dx, dg = np.empty_like(x), np.empty_like(x)
    for t in range(s["longest"] - 1, -1, -1):
        q = order[: live[t]]
        k = head[q] + up * t
        lam = dh[k] + mu[q]
        if t:
            before = h[k - up]
        else:
            before = 0.0 if h0 is None else h0[q]
        dx[k] = rest[k] * lam
        dg[k] = a[k] * rest[k] * lam * (before - x[k]) if sig else lam * before
        mu[q] = a[k] * lam
    dg = dg.reshape(len(dg), -1, case["group"]).sum(2)
    return (torch.from_numpy(dg), torch.from_numpy(dx),
            None if h0 is None else torch.from_numpy(mu))
