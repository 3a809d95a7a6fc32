"""The sequence operators at the limits of what a launch, a tag or a format holds, and
the variants of their kernels that sizes choose."""
import ctypes

import numpy as np
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


# What the entry points hand to the launches, for calls whose workspace is made here.
class RecCall(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                "gate x h dh h0 init offsets out dgate fin flag".split()] + \
               [(n, ctypes.c_int64) for n in "ld_gate ld_x ld_h ld_dh ld_out ld_dgate".split()] + \
               [(n, ctypes.c_int) for n in "tokens nseq D group offset_bytes down".split()]


class ScanSpace(ctypes.Structure):
    _fields_ = [("head", ctypes.c_void_p), ("counters", ctypes.c_int),
                ("flags", ctypes.c_size_t), ("words", ctypes.c_size_t)]


class Launch(ctypes.Structure):
    _fields_ = [("stream", ctypes.c_void_p), ("owner", ctypes.c_void_p), ("take", ctypes.c_void_p)]


def logits_call(pg):  # noqa: F811
    class LogitsCall(ctypes.Structure):
        _fields_ = [("a", pg.LogitsArgs), ("flag", ctypes.c_void_p), ("tiles", ctypes.c_int),
                    ("head", ctypes.c_void_p), ("words", ctypes.c_void_p),
                    ("stride", ctypes.c_int64)]
    return LogitsCall


INTERNAL = 2  # kFlagInternal
LINE = 16     # kHeadLine


def test_a_ticket_past_the_chunks(pg, ctx):  # noqa: F811
    """A tile whose counter another call has moved: its workgroups say so and touch
    nothing, the other tile is what it is."""
    lib = pg.load_library()
    space = lib._ZN2pg10scan_spaceEli
    space.argtypes, space.restype = [ctypes.c_int64, ctypes.c_int], ScanSpace
    launch = lib._ZN2pg17launch_recurrenceERKNS_7RecCallEiibRKNS_9ScanSpaceERKNS_6LaunchE
    launch.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_bool, ctypes.c_void_p,
                       ctypes.c_void_p]
    q = Seqs("f32", [600], 64, 1, True, seed=32)
    off = q.offsets()
    want, _ = ctx.recurrence(q.gate, q.x, off, h0=q.h0)
    sp = space(600, 64)
    n = sp.counters * LINE + sp.flags + sp.words
    for ticket in (5, 6, 1 << 31, (1 << 32) - 6):  # of five chunks of 128 tokens
        room = torch.zeros(n, dtype=torch.int64, device="cuda")
        room[:sp.counters * LINE:LINE] = 1 << 32
        room[0] += ticket
        before = room.clone()
        h = torch.full_like(q.x, 7.0)
        flag = torch.zeros(3, dtype=torch.int32, device="cuda")
        sp.head = room.data_ptr()
        call = RecCall(gate=q.gate.data_ptr(), x=q.x.data_ptr(), h0=q.h0.data_ptr(),
                       init=q.h0.data_ptr(), offsets=off.data_ptr(), out=h.data_ptr(),
                       flag=flag.data_ptr(), ld_gate=64, ld_x=64, ld_out=64, tokens=600, nseq=1,
                       D=64, group=1, offset_bytes=4)
        on = Launch(stream=torch.cuda.current_stream().cuda_stream)
        assert launch(ctypes.byref(call), pg.F32, pg.GATE_SIGMOID, False, ctypes.byref(sp),
                      ctypes.byref(on)) == 0
        torch.cuda.synchronize()
        assert flag.tolist() == [INTERNAL, 0, 0]
        assert (h[:, :32] == 7).all() and torch.equal(h[:, 32:], want[:, 32:])
        # of the first tile only the counter moved, by its five workgroups
        assert int(room[0] - before[0]) == 5
        flags = slice(sp.counters * LINE, sp.counters * LINE + 5 + 1)
        assert torch.equal(room[flags], before[flags])
        words = sp.counters * LINE + sp.flags
        first = slice(words, words + 8 * (8 * 5 + 12 * 1))
        assert torch.equal(room[first], before[first])


def test_more_parts_than_a_row_has(pg, ctx):  # noqa: F811
    lib = pg.load_library()
    launch = lib._ZN2pg13launch_logitsENS_10LogitsCallERKNS_6LaunchE
    LogitsCall = logits_call(pg)
    launch.argtypes = [LogitsCall, ctypes.c_void_p]
    V = 2000  # two parts
    x = torch.randn(2, V, device="cuda")
    head = torch.zeros(2 * LINE, dtype=torch.int64, device="cuda")
    head[::LINE] = 1 << 32
    head[0] += 2
    words = torch.zeros(2 * 2 * 3, dtype=torch.int64, device="cuda")
    flag = torch.zeros(3, dtype=torch.int32, device="cuda")
    token = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    call = LogitsCall(flag=flag.data_ptr(), head=head.data_ptr(), words=words.data_ptr(), stride=2)
    call.a = pg.LogitsArgs(logits=x.data_ptr(), token=token.data_ptr(), ld_logits=V, rows=2, V=V)
    on = Launch(stream=torch.cuda.current_stream().cuda_stream)
    assert launch(call, ctypes.byref(on)) == 0
    torch.cuda.synchronize()
    assert flag.tolist() == [INTERNAL, 0, 0]
    assert token.tolist() == [-7, int(x[1].argmax())]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [5, 64])
def test_dropout_of_table_rows_keeps_the_sign_of_zero(ctx, dtype, d):  # noqa: F811
    """Rows taken by their ids are the bits that the same rows give without ids."""
    rng = np.random.default_rng(d)
    table = dev(np.where(rng.random((40, d)) < 0.5, -0.0, rng.normal(size=(40, d))), dtype)
    ids = torch.from_numpy(rng.integers(0, 40, 300).astype(np.int32)).cuda()
    rows = table[ids.long()]
    bits = lambda t: t.view(torch.int32 if dtype == "f32" else torch.int16)  # noqa: E731
    assert torch.equal(bits(ctx.dropout(table, 0.0, 3, ids=ids)), bits(rows))
    assert torch.equal(bits(ctx.dropout(table, 0.4, 3, ids=ids)), bits(ctx.dropout(rows, 0.4, 3)))
    add = torch.full_like(rows, -0.0)
    assert torch.equal(bits(ctx.dropout(table, 0.4, 3, ids=ids, add=add)),
                       bits(ctx.dropout(rows, 0.4, 3, add=add)))


# The rules by which the launches choose a variant, written out again: a case below says
# which one it is there for, and fails if a change of the rules moves it to another.


def scan_variant(dtype, sig, grad, tokens, D, group):
    """Lanes of a row of threads and tokens of a thread."""
    size = 4 if dtype == "f32" else 2
    per_group = -(-group // 4) if group > 1 else 1
    lanes = per_group * (D // group) if group > 1 else -(-D // 4)
    usual = 3 if D <= 64 or (size == 4 and D <= 512) else 4
    log2 = 3
    while log2 < 6 and 1 << log2 < lanes and (log2 < usual or 1 << log2 < per_group):
        log2 += 1
    row = 1 << log2
    tiles = -(-(D // group) // (row // per_group)) if group > 1 else -(-D // (4 * row))
    long = (12 if grad else 16) if size == 2 else 8 if grad else 12 if sig else 16
    chunks = max(1, -(-tokens // (256 // row * long)))
    return row, long if chunks * tiles >= 256 else 4


LONG_CHUNKS = [(dtype, sig, D, group, row)
               for dtype in ("f32", "bf16", "f16")
               for sig, D, group, row in (
                   (True, 512, 1, 8 if dtype == "f32" else 16),
                   (False, 512, 1, 8 if dtype == "f32" else 16),
                   (dtype != "bf16", 509, 1, 8 if dtype == "f32" else 16),
                   (True, 512, 64, 16), (False, 512, 64, 16), (dtype == "bf16", 510, 5, 8 if dtype == "f32" else 16),
                   (dtype != "f16", 512, 128, 32), (dtype == "f16", 512, 256, 64))]


@pytest.mark.parametrize("dtype,sig,D,group,row", LONG_CHUNKS)
def test_recurrence_with_long_chunks(pg, ctx, dtype, sig, D, group, row):  # noqa: F811
    """Threads with the most tokens they take, forward and gradient: sequences that begin and
    end in every place of a chunk, and one that goes through many."""
    tokens = 8300
    most = 16 if dtype != "f32" else 12 if sig else 16
    assert scan_variant(dtype, sig, False, tokens, D, group) == (row, most)
    assert scan_variant(dtype, sig, True, tokens, D, group) == (row, 12 if dtype != "f32" else 8)
    rng = np.random.default_rng([D, group, sig])
    lengths = np.concatenate([rng.integers(0, 40, 60), [3200], rng.integers(100, 300, 6), [0, 1]])
    lengths = np.append(lengths, tokens - lengths.sum())
    Seqs(dtype, lengths, D, group, sig, state=group != 128, seed=33).check(ctx, pg, not sig)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("empty", [1023, 1024, 1025, 2049, 3000])
def test_recurrence_of_many_empty_sequences_at_one_place(pg, ctx, empty, reverse):  # noqa: F811
    """More offsets within reach of a chunk than are read at a time."""
    none = [0] * empty
    for lengths in (none + [5] + none + [700] + [1] * 40 + none, [300] + none + [300], none):
        for state in (True, False):
            Seqs("f32", lengths, 12, 1, True, state=state, seed=34).check(
                ctx, pg, reverse, torch.int64 if empty % 2 else torch.int32)


@pytest.mark.parametrize("nseq", [1039, 1040, 1104, 4223, 4224, 4225, 4289])
def test_recurrence_finds_its_first_offset(pg, ctx, nseq):  # noqa: F811
    """Counts on both sides of those that the search's 65 parts divide."""
    Seqs("f32", [1] * nseq, 8, 1, True, seed=35).check(ctx, pg, nseq % 2 == 0)


def scores_variant(rows, V):
    words = 32
    while words > 4 and rows * -(-V // (words * 256)) < 512:
        words //= 2
    return words


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cap", [300, 33_000])
@pytest.mark.parametrize("rows,V,words", [
    (48, 32_003, 8), (48, 32_767, 8), (48, 32_769, 8), (64, 35_003, 16), (64, 36_863, 16),
    (64, 36_865, 16), (64, 65_535, 32), (64, 65_537, 32), (30, 16_384, 4), (64, 20_479, 8)])
def test_scores_with_every_length_of_a_part(ctx, dtype, cap, rows, V, words):  # noqa: F811
    """Parts of 1,024 to 8,192 words with counters of 16 and 32 bits; vocabularies just
    below and just above whole parts."""
    assert scores_variant(rows, V) == words
    kind = (rows + V + cap) % 3
    Scores(dtype, rows, V, cap=cap, masks=(rows, 1, rows + 2)[kind], bias=("shared", "rows")[V % 2],
           seed=36).check(ctx)
