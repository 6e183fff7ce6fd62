"""Every row that a query sees is weighed once, however the calls of blocks of queries divide the rows.

With queries of zeros every weight is 1 / (rows seen), and with values of 0 and 1 the sums are whole numbers below 2^24, exact in any
order: an output is its row count, times the reciprocal of the number seen, rounded.  Tolerance: the reciprocal and the product 2^-24 each
of the result, the output's rounding 2^-8 (bf16) or 2^-24 (f32) of it; zeros are exact.  In the values' first d - 16 elements a tile of
32 rows counts for element `tile % (d - 16)`: of 141,000 rows (d = 64) each has 92 tiles, so that one that is lost or weighed twice moves it
by 1.08%, which a rounding of 0.39% does not bring back within the tolerance of 0.39%.  Each of the last 16 elements belongs to one
row of the sequence (the first, the last, others anywhere): losing or repeating it changes that output by its whole size."""
import numpy as np
import pytest
import torch

from test_gpu_q4 import DT, Cache, gen, i32
from test_gpu_q4_window import seen_of

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2609_03515_amd.binding")


def content(n, hkv, d, seed):
    """Values [hkv][n][d] of 0 and 1."""
    x = torch.zeros(hkv, n, d)
    r = torch.arange(n)
    x[:, r, r // 32 % (d - 16)] = 1.0
    for h in range(hkv):
        some = torch.randperm(n, generator=gen(100 * seed + h))
        some = torch.cat((torch.tensor([0, n - 1] if n > 1 else [0] * n, dtype=torch.int64), some[(some != 0) & (some != n - 1)]))[:16]
        x[h, some, d - 16 + torch.arange(len(some))] = 1.0
    return x


def filled(lens, seed=3, **kw):
    """A cache of such values under random keys, the same in every layer; t.rows: the values of every slot."""
    t = Cache(lens, **kw)
    most = max(lens)
    t.rows = [content(n, t.hkv, t.d, seed + b) for b, n in enumerate(lens)]
    v = torch.zeros(1, len(lens), t.hkv, most, t.d)
    for b, n in enumerate(lens):
        v[0, b, :, :n] = t.rows[b]
    k = torch.randn(1, len(lens), t.hkv, most, t.d, generator=gen(seed + 77))
    k, v = k.to(DT[t.dtype]).cuda(), v.to(DT[t.dtype]).cuda()
    for l in range(t.layers):
        B.kv_q4_store(t.c, l, 1, most, k, v, t.ws, count=t.c.len)
    assert t.faults() == 0
    return t


def same_counts(t, got, rows, seen):
    """got [hq][m][d]: outputs of queries of zeros that see seen [m][n] of the rows."""
    sums = np.matmul(seen.astype(np.float32), rows.numpy())  # (whole numbers below 2^24: exact)
    want = np.repeat(sums.astype(np.float64) / np.maximum(seen.sum(-1), 1)[None, :, None], t.hq // t.hkv, axis=0)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= want * (1.01 * 2.0 ** -8 if t.dtype == "bf16" else 2.0 ** -22)).all(), (err.max(), np.argwhere(err > want * 2.0 ** -7)[:5].tolist())


# ---- samples of a full table ---------------------------------------------------------------------------------------------------

def shared_call(t, group, layers=None):
    layers = layers or t.layers
    q = torch.zeros(layers, t.shape.batch, t.hq, t.d, dtype=DT[t.dtype], device="cuda")
    o = torch.full_like(q, 9.0)
    ws = B.q4_shared_workspace(t.shape, t.cap, layers)
    B.kv_q4_attend_shared(t.c, 0, layers, t.cap, i32(group), q, o, ws)
    lens = t.c.len.tolist()
    for l in {0, layers - 1}:
        for b, n in enumerate(lens):
            same_counts(t, o[l, b][:, None], t.rows[b][:, :n], np.ones((1, n), dtype=bool))
    assert B.faults(ws, clear=True) == 0


@pytest.mark.parametrize("dtype,fan", [("bf16", 1), ("bf16", 6), ("bf16", 17), ("f32", 5)])
@pytest.mark.parametrize("page_rows,pages", [(16, 1), (16, 2), (16, 10), (16, 528), (32, 1), (32, 5), (64, 3), (64, 132), (128, 1), (128, 2), (128, 66), (256, 1), (256, 33)])
def test_full_tables(page_rows, pages, dtype, fan):
    """Slots that fill their tables to the last row, sharing all pages."""
    n, batch = page_rows * pages, fan + 1
    t = filled([n] + [0] * fan, hq=4, hkv=1, page_rows=page_rows, max_pages=pages, d=64, dtype=dtype)
    B.kv_q4_fork(t.c, i32([0] * fan), i32(list(range(1, batch))), t.ws)
    assert t.faults() == 0 and t.c.len.tolist() == [n] * batch and t.cap == n
    t.rows = t.rows[:1] * batch
    shared_call(t, [0] * batch)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page_rows,pages", [(16, 2), (16, 11), (32, 5), (64, 40), (256, 1), (256, 12)])
def test_a_full_table_beside_shorter_slots(page_rows, pages, dtype):
    n = page_rows * pages
    for full in (0, 3, 7):
        lens = [min(n, 1 + 37 * i) for i in range(8)]
        lens[full] = n
        t = filled(lens, hq=8, hkv=2, page_rows=page_rows, max_pages=pages, dtype=dtype)
        shared_call(t, [0] * 8)
        shared_call(t, [i % 2 for i in range(8)])


def test_full_tables_of_many_layers():
    """Enough layers and heads for workgroups of eight waves."""
    t = filled([256, 128, 255, 256, 200, 1, 256, 256], layers=64, hq=16, hkv=4, page_rows=32, max_pages=8, d=64)
    shared_call(t, [0] * 8)
    t = filled([256] * 70, layers=8, hq=16, hkv=4, page_rows=64, max_pages=4, d=64)
    shared_call(t, [i % 3 for i in range(70)])


# ---- windows, and the marks of the tiles that a block sees any row of ----------------------------------------------------------------

def placed(t, places, rows):
    """The rows' positions: none kept, in order, with gaps and some out of order under the newest `rows`, or (any) Cache's random order."""
    if places == "rows":
        t.c.pos = None
    elif places == "ordered":
        t.c.pos.copy_(torch.arange(t.cap, dtype=torch.int32).expand(len(t.lens), t.cap))
    elif places == "evicted":
        for b, n in enumerate(t.lens):
            old = max(0, n - rows)
            p = 3 * torch.arange(old) + torch.randint(0, 3, (old,), generator=gen(b))
            swap = torch.randperm(old, generator=gen(b + 50))[: old // 8]
            p[swap] = p[swap.flip(0)]
            t.c.pos[b, :old] = p.to(torch.int32)
            t.c.pos[b, old:n] = torch.arange(3 * old, 3 * old + n - old, dtype=torch.int32)
    return t


def window_call(t, rows, counts, window, sinks, layers=None, vectors=None, n_max=None, faults=0):
    """vectors: the queries of a block where the call makes marks, which are in the workspace behind its first 256 bytes: 64 tiles to a
    word, [slot][block][word].  A slot of which counts says None cannot be: zeros."""
    layers, n_max = layers or t.layers, n_max or t.cap
    lens = t.c.len.tolist()
    q = torch.zeros(layers, len(lens), t.hq, rows, t.d, dtype=DT[t.dtype], device="cuda")
    o = torch.full_like(q, 9.0)
    ws = B.q4_window_workspace(t.shape, n_max, rows, layers)
    ws[256:] = 77
    B.kv_q4_attend_window(t.c, 0, layers, n_max, rows, q, o, ws, window=window, sinks=sinks, count=i32([rows + 1 if m is None else m for m in counts]))
    blocks, words = -(-rows // (vectors or rows)), -(-n_max // 2048)
    marks = ws[256 : 256 + 8 * len(lens) * blocks * words].cpu().numpy().view(np.uint64).reshape(len(lens), blocks, words)
    for b, (n, m) in enumerate(zip(lens, counts)):
        if m is None:
            assert (o[:, b] == 0).all() and (not vectors or (marks[b] == 0).all())
            continue
        pos = np.arange(n) if t.c.pos is None else t.c.pos[b, :n].cpu().numpy().astype(np.int64)
        seen = seen_of(pos, n, m, window, sinks)
        for l in {0, layers - 1}:
            assert (o[l, b, :, m:] == 9.0).all()
            same_counts(t, o[l, b, :, :m], t.rows[b][:, :n], seen)
        for k in range(0, m if vectors else 0, vectors or 1):
            # (of a block's queries together: up to the last of their positions, from the first one's window on, and the sinks)
            at = pos[n - m + k : n - m + min(k + vectors, m)]
            some = (pos <= at.max()) & ((pos > at.min() - window) | (pos < sinks) | (window == 0))
            bits = np.pad(some, (0, words * 2048 - n)).reshape(-1, 32).any(1)
            assert np.array_equal(marks[b, k // vectors], np.packbits(bits, bitorder="little").view(np.uint64)), (b, k)
    assert B.faults(ws, clear=True) == faults


@pytest.mark.parametrize("dtype,window,vectors", [("bf16", 0, 16), ("bf16", 50, 8), ("f32", 0, 4), ("f32", 50, 4)])
def test_marks_of_slots_that_cannot_be(dtype, window, vectors):
    """Bad lengths and counts in every slot, the first among them, of a call that marks tiles."""
    rows, page_rows = 70, 64
    t = filled([90, 300, 90, 96, 130], hq=16, hkv=4, d=64, page_rows=page_rows, max_pages=131072 // page_rows, dtype=dtype)
    # (positions inside a larger buffer)
    around = torch.zeros(len(t.lens) * t.cap + 2 * 4096, dtype=torch.int32, device="cuda")
    inner = around[4096 : 4096 + len(t.lens) * t.cap].view(len(t.lens), t.cap)
    inner.copy_(t.c.pos)
    t.c.pos = inner
    good = [70, 70, 1, 50, 70]
    window_call(t, rows, good, window, 9, vectors=vectors)
    for bad in ([0], [0, 1, 4], [0, 1, 2, 3, 4]):
        window_call(t, rows, [None if b in bad else m for b, m in enumerate(good)], window, 9, vectors=vectors, faults=B.KV_FAULT_CACHE)
    t.c.len[0], t.c.len[3] = -3, t.cap + 1
    window_call(t, rows, [None, 70, 1, None, 70], window, 9, vectors=vectors, faults=B.KV_FAULT_CACHE)


DECODE, CHUNK = ((0, 0), (700, 40), (5, 0)), ((0, 0), (1000, 3))


@pytest.mark.parametrize("places", ["rows", "ordered", "evicted"])
@pytest.mark.parametrize("dtype,hq,hkv,d,layers,lens,page_rows,rows,windows", [
    ("bf16", 4, 1, 128, 1, [9001, 400, 5000], 64, 1, DECODE), ("f32", 4, 1, 64, 1, [9001, 400, 5000], 64, 1, DECODE),
    ("bf16", 2, 1, 64, 1, [141_000], 256, 1, ((0, 0), (40_000, 100))), ("f32", 4, 1, 64, 1, [9001, 400, 5000], 32, 70, CHUNK),
    ("bf16", 4, 1, 128, 1, [9001, 400, 5000], 64, 70, CHUNK), ("bf16", 4, 1, 64, 1, [141_000], 256, 24, ((0, 0), (40_000, 100))),
    ("bf16", 14, 2, 64, 2, [9001, 8999], 16, 130, CHUNK), ("bf16", 32, 8, 64, 1, [32_749], 128, 128, ((0, 0), (30_000, 5))),
    ("bf16", 32, 8, 128, 8, [4100], 64, 128, ((0, 0),))])
def test_every_row_once(dtype, hq, hkv, d, layers, lens, page_rows, rows, windows, places):
    """One, two and four column tiles, blocks divided among workgroups, waves of many runs of 64 tiles."""
    t = placed(filled(lens, dtype=dtype, hq=hq, hkv=hkv, d=d, layers=layers, page_rows=page_rows), places, rows)
    for window, sinks in windows:
        window_call(t, rows, [min(rows, n) for n in lens], window, sinks)


@pytest.mark.parametrize("places", ["ordered", "evicted", "any"])
@pytest.mark.parametrize("dtype,hq,hkv,layers,lens,page_rows,rows,window,vectors", [
    ("bf16", 16, 4, 2, [9001, 7777, 2049], 64, 130, 40, 8), ("bf16", 16, 4, 2, [9001, 7777, 2049], 64, 260, 0, 16), ("bf16", 16, 4, 2, [9001, 0, 7777], 16, 400, 5000, 16),
    ("f32", 16, 4, 2, [9001, 4100], 64, 130, 0, 4), ("bf16", 16, 1, 1, [9001, 2048], 256, 1000, 0, 4), ("bf16", 16, 1, 1, [9001, 2048], 256, 300, 0, None),
    ("bf16", 2, 1, 1, [141_000], 256, 24, 128, 16), ("f32", 2, 1, 1, [141_000], 256, 24, 128, 8), ("bf16", 4, 2, 1, [141_000], 128, 600, 100_000, 32),
    ("bf16", 2, 2, 1, [141_000], 256, 1100, 100_000, 64)])
def test_marks(dtype, hq, hkv, layers, lens, page_rows, rows, window, vectors, places):
    """Marks of many words, past 131,072 rows among them, and every row that a query sees found by them once (vectors None: divided among
    so many workgroups that the waves look for themselves)."""
    t = placed(filled(lens, dtype=dtype, hq=hq, hkv=hkv, d=64, layers=layers, page_rows=page_rows), places, rows)
    counts = [min(rows, n) for n in lens]
    window_call(t, rows, counts, window, 9, vectors=vectors)
    window_call(t, rows, [max(0, c - 7 * i - 3) for i, c in enumerate(counts)], window, 9, vectors=vectors)


@pytest.mark.parametrize("places", ["rows", "any"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page_rows,pages", [(16, 1), (16, 2), (16, 528), (64, 3), (256, 1), (256, 33)])
def test_full_tables_in_windows(page_rows, pages, dtype, places):
    """Slots that fill their tables to the last row, beside an empty and a short one."""
    n = page_rows * pages
    t = placed(filled([n, 0, min(n, 9)], hq=4, hkv=1, d=64, page_rows=page_rows, max_pages=pages, dtype=dtype), places, 9)
    for rows in (1, 9, 70):
        for window, sinks in ((0, 0), (20, 3)):
            window_call(t, rows, [min(rows, n), 0, min(rows, n, 9)], window, sinks)


# ---- samples of long prompts ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,fan,hq,hkv,layers", [("bf16", 2, 4, 1, 1), ("bf16", 15, 4, 1, 1), ("bf16", 11, 28, 4, 2), ("f32", 5, 4, 1, 1), ("bf16", 15, 32, 8, 32)])
@pytest.mark.parametrize("page_rows", [16, 128])
def test_long_prompts_rows_once(dtype, fan, hq, hkv, layers, page_rows):
    """Pages that all samples share, and ends of different samples inside them."""
    n, batch = 9001 if layers < 32 else 2049, fan + 1
    t = filled([n] + [0] * fan, dtype=dtype, hq=hq, hkv=hkv, d=64, layers=layers, page_rows=page_rows)
    B.kv_q4_fork(t.c, i32([0] * fan), i32(list(range(1, batch))), t.ws)
    t.rows = t.rows[:1] * batch
    shared_call(t, [0] * batch)
    shared_call(t, [b % 2 for b in range(batch)])
    t.c.len.copy_(i32([n - (311 * b if b % 3 else b) for b in range(batch)]) if layers < 32 else i32([n - 97 * b for b in range(batch)]))
    shared_call(t, [0] * batch)


# ---- the forms that keep all of a probability -------------------------------------------------------------------------------------

@pytest.mark.parametrize("hq,hkv,rows", [(4, 4, 16), (4, 2, 8), (6, 2, 5), (4, 1, 4), (7, 1, 2), (8, 1, 2)])
@pytest.mark.parametrize("places", ["rows", "ordered"])
@pytest.mark.parametrize("d", [64, 128])
def test_few_queries_are_exact(hq, hkv, rows, places, d):
    """bf16 queries that fit one column tile: the bound of a single query, without the rounding of probabilities."""
    from test_gpu_q4_window import limits, reference

    lens = [33, 700, 150, 16]
    t = placed(Cache(lens, hq=hq, hkv=hkv, d=d, page_rows=32).fill(), places, rows)
    q = torch.randn(1, 4, hq, rows, d, generator=gen(7)).bfloat16().cuda()
    o = torch.full_like(q, 9.0)
    ws = B.q4_window_workspace(t.shape, t.cap, rows, 1)
    for window, sinks in ((0, 0), (24, 3)):
        B.kv_q4_attend_window(t.c, 0, 1, t.cap, rows, q, o, ws, window=window, sinks=sinks)
        for b, n in enumerate(lens):
            k, v = t.values(0, b)
            want, size, av = reference(q[0, b].double().cpu().numpy(), k, v, seen_of(np.arange(n), n, rows, window, sinks))
            err, lim = np.abs(o[0, b].double().cpu().numpy() - want), limits(t, want, size, av, n, 1)
            assert (err <= lim).all(), (b, (err / lim).max())


@pytest.mark.parametrize("hq,hkv,batch", [(4, 4, 16), (4, 2, 8), (6, 2, 5), (4, 1, 4), (7, 1, 2), (16, 1, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_few_samples_are_exact(hq, hkv, batch, d):
    """bf16 samples that fit one column tile, likewise."""
    from test_gpu_q4_window import limits, reference

    n = 700
    t = Cache([n] + [0] * (batch - 1), hq=hq, hkv=hkv, d=d, page_rows=32).fill()
    if batch > 1:
        B.kv_q4_fork(t.c, i32([0] * (batch - 1)), i32(list(range(1, batch))), t.ws)
    q = torch.randn(1, batch, hq, d, generator=gen(7)).bfloat16().cuda()
    o = torch.full_like(q, 9.0)
    B.kv_q4_attend_shared(t.c, 0, 1, t.cap, i32([0] * batch), q, o, B.q4_shared_workspace(t.shape, t.cap, 1))
    k, v = t.values(0, 0)
    for b in range(batch):
        want, size, av = reference(q[0, b].double().cpu().numpy()[:, None], k, v, np.ones((1, n), dtype=bool))
        err, lim = np.abs(o[0, b].double().cpu().numpy()[:, None] - want), limits(t, want, size, av, n, 1)
        assert (err <= lim).all(), (b, (err / lim).max())


# ---- bytes that no store writes --------------------------------------------------------------------------------------------------

def scribble(t, b, rows, keys=True, seed=5):
    """Any codes, and scale bytes of every kind, into rows of a slot: values, and keys."""
    pool = t.c.pool.cpu().view(t.layers, t.shape.n_pages, t.hkv, -1)
    pr, d, r = t.shape.page_rows, t.d, np.random.RandomState(seed)
    half = pr * (d // 2 + d // 32)
    for i in rows:
        page = int(t.c.table[b, i // pr])
        for first in ([0, half] if keys else [half]):
            c, e = first + i % pr * (d // 2), first + pr * (d // 2) + i % pr * (d // 32)
            shape = (t.layers, t.hkv)
            pool[:, page, :, c : c + d // 2] = torch.from_numpy(r.randint(0, 256, shape + (d // 2,)).astype(np.uint8))
            pool[:, page, :, e : e + d // 32] = torch.from_numpy(r.choice([253, 254, 255, 252, 130, 0], shape + (d // 32,)).astype(np.uint8))
    t.c.pool.copy_(pool.view(-1))


FORMS = [("bf16", 128, 1, 0), ("bf16", 128, 20, 0), ("bf16", 64, 20, 0), ("bf16", 128, 70, 1 << 17), ("bf16", 64, 70, 1 << 17), ("f32", 128, 20, 0), ("f32", 64, 1, 0)]


@pytest.mark.parametrize("dtype,d,rows,room", FORMS)
@pytest.mark.parametrize("places", ["rows", "ordered"])
def test_masked_rows_of_any_bytes(dtype, d, rows, room, places):
    """Rows before the window and rows that are not stored yet hold anything, and the queries that do not see them are as without."""
    from test_gpu_q4_window import limits, reference

    n = 200
    t = placed(Cache([n], hq=8, hkv=2, d=d, dtype=dtype, page_rows=32, max_pages=room // 32 or 8).fill(), places, rows)
    later = 0 if rows == 1 else rows // 2  # of the newest rows, those that are not stored
    old = n - rows - 40                    # before the first query's window
    scribble(t, 0, list(range(n - later, n)) + list(range(old)))
    q = torch.randn(1, 1, 8, rows, d, generator=gen(2)).to(DT[dtype]).cuda()
    o = torch.full_like(q, 9.0)
    ws = B.q4_window_workspace(t.shape, t.cap, rows, 1)
    B.kv_q4_attend_window(t.c, 0, 1, t.cap, rows, q, o, ws, window=40)
    m = rows - later
    pos = np.arange(n)
    seen = seen_of(pos, n, rows, 40, 0)[:m]
    assert seen.any(1).all() and not seen[:, :old].any() and not seen[:, n - later :].any()
    k, v = t.values(0, 0)
    want, size, av = reference(q[0, 0, :, :m].double().cpu().numpy(), k, v, seen)
    err, lim = np.abs(o[0, 0, :, :m].double().cpu().numpy() - want), limits(t, want, size, av, n, rows)
    assert (err <= lim).all(), (np.nanmax(err), np.isnan(err).any())


@pytest.mark.parametrize("dtype,d,rows,room", FORMS)
def test_rows_seen_of_any_bytes(dtype, d, rows, room):
    """A query that sees one row gives its values, whatever else its tile holds: numbers up to 1.5 2^127, infinities past that (2^128 is
    neither a bf16 nor an f32 number), NaN for byte 255."""
    n = 200
    t = Cache([n], hq=8, hkv=2, d=d, dtype=dtype, page_rows=32, max_pages=room // 32 or 8).fill()
    t.c.pos = None
    scribble(t, 0, range(n), keys=False)
    q = torch.randn(1, 1, 8, rows, d, generator=gen(2)).to(DT[dtype]).cuda()
    o = torch.full_like(q, 9.0)
    ws = B.q4_window_workspace(t.shape, t.cap, rows, 1)
    B.kv_q4_attend_window(t.c, 0, 1, t.cap, rows, q, o, ws, window=1)
    v = np.repeat(t.values(0, 0)[1][:, n - rows :], 4, axis=0)
    want = np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)
    got = o[0, 0].double().cpu().numpy()
    plain = np.isfinite(want)
    assert np.array_equal(np.where(plain, 0.0, got), np.where(plain, 0.0, want), equal_nan=True)
    # A weight of the one row is 1 within the logit's error, 2^-22 of it, and a few roundings; codes times scales are bf16 numbers.
    # Numbers below the smallest normal one, 2^-126, may be 0.  And where the tile holds a byte above 252, its values are added in
    # quarters and the sum is taken four times: a scale of byte 0 or 1 has no quarter above the smallest scale, 2^-127, so that
    # x = code 2^-127 or code 2^-126 becomes 4 code 2^-127: off by at most (4 - 1) 6 2^-127 = 2^-122.8.
    err, size = np.abs(np.where(plain, got, 0.0) - np.where(plain, want, 0.0)), np.abs(np.where(plain, want, 0.0))
    assert (err <= (2.0 ** -17 if dtype == "f32" else 0.0) * size + 2.0 ** -126 + (size < 6.1 * 2.0 ** -126) * 18 * 2.0 ** -127).all()


@pytest.mark.parametrize("dtype,d,fan,layers", [("bf16", 128, 1, 1), ("bf16", 128, 12, 1), ("bf16", 64, 12, 1), ("bf16", 64, 7, 128), ("f32", 128, 5, 1), ("f32", 64, 5, 1)])
def test_other_samples_rows_of_any_bytes(dtype, d, fan, layers):
    """Pages that one sample has for itself hold anything; the other samples' outputs are as without."""
    from test_gpu_q4_window import limits, reference

    n, batch = 96, fan + 1
    t = Cache([n] + [n] * fan, hq=8, hkv=2, d=d, dtype=dtype, page_rows=32, layers=layers).fill()
    # the first page of all is the first slot's; slot 1's others hold anything
    t.c.table[:, 0] = t.c.table[0, 0]
    scribble(t, 1, range(32, 96))
    q = torch.randn(layers, batch, 8, d, generator=gen(2)).to(DT[dtype]).cuda()
    o = torch.full_like(q, 9.0)
    ws = B.q4_shared_workspace(t.shape, t.cap, layers)
    B.kv_q4_attend_shared(t.c, 0, layers, t.cap, i32([0] * batch), q, o, ws)
    for l in {0, layers - 1}:
        for b in range(batch):
            if b == 1:
                continue
            k, v = t.values(l, b)
            want, size, av = reference(q[l, b].double().cpu().numpy()[:, None], k, v, np.ones((1, n), dtype=bool))
            err, lim = np.abs(o[l, b].double().cpu().numpy()[:, None] - want), limits(t, want, size, av, n, 2)
            assert (err <= lim).all(), (l, b, np.nanmax(err), np.isnan(err).any())
