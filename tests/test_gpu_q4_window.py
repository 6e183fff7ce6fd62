"""kv_q4_attend_window against the definition in float64.

Tolerances.  Logits: products of a query (bf16: exact; f32: three parts, 24 bits) and a stored element (2 bits), d of them added in
32 bits, are off by at most (d + 4) 2^-24 sum |q k| / sqrt(d), their scaling by 2^-23 of itself; a probability by twice the logits'
error, plus the sums over n rows and the exponential (n + 64) 2^-24, all relative to sum a |v|.  bf16 calls round the output (2^-8 of
itself), and those of several queries may round each probability to bf16: weights a (1 + e) / sum a (1 + e') with |e|, |e'| <= 2^-8 are
off by 2^-7 (and 2^-15 for the second order) of sum a |v|."""
import numpy as np
import pytest
import torch

import q4_reference as R
from test_gpu_q4 import DT, HEADS, Cache, gen, i32

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2609_03515_amd.binding")


def reference(q, k, v, seen):
    """q [hq][m][d], k, v [hkv][n][d], seen [m][n] -> outputs [hq][m][d], the largest sum |q k| / sqrt(d), sum a |v|."""
    hq, m, d = q.shape
    kk, vv = np.repeat(k, hq // k.shape[0], axis=0), np.repeat(v, hq // v.shape[0], axis=0)
    size = 0.0
    out, av = np.zeros((hq, m, d)), np.zeros((hq, m, d))
    for h in range(hq):
        # rows that no query of the call sees take no part, whatever they hold
        use = seen.any(0)
        if not use.any():
            continue
        kh, vh, s = kk[h][use], vv[h][use], seen[:, use]
        z = np.where(s, q[h] @ kh.T / np.sqrt(d), -np.inf)
        size = max(size, np.nanmax(np.abs(q[h]) @ np.abs(kh).T) / np.sqrt(d))
        top = z.max(-1, keepdims=True)
        e = np.exp(z - np.where(np.isfinite(top), top, 0.0))
        total = e.sum(-1, keepdims=True)
        a = e / np.where(total > 0, total, 1.0)
        out[h], av[h] = a @ vh, a @ np.abs(vh)
    return out, size, av


def seen_of(pos, n, m, window, sinks):
    """[m][n]: the rows that the queries of the newest m rows see."""
    p = pos[:n].astype(np.int64)
    at = p[n - m :, None]
    s = p[None] <= at
    return s & ((p[None] > at - window) | (p[None] < sinks)) if window else s


def limits(t, want, size, av, n, rows):
    rel = 2 * ((t.d + 4) * 2.0 ** -24 * size + 2.0 ** -22 * size) + (n + 64) * 2.0 ** -24
    if t.dtype == "bf16":
        return 2.0 ** -8 * np.abs(want) * 1.01 + (rel + (2.0 ** -7 + 2.0 ** -15 if rows > 1 else 0.0)) * av * 1.01
    return (rel + 2.0 ** -23) * av


def run(t, rows, counts, window, sinks, layers=None, layer0=0, n_max=None, left=9.0, ws=None, q=None):
    layers = layers or t.layers
    if q is None:
        q = torch.randn(layers, len(t.lens), rows, t.hq, t.d, generator=gen(7)).to(DT[t.dtype]).cuda().transpose(2, 3)
    o = torch.full((layers, len(t.lens), rows, t.hq, t.d), left, dtype=DT[t.dtype], device="cuda").transpose(2, 3)
    ws = t.wws if ws is None else ws
    B.kv_q4_attend_window(t.c, layer0, layers, n_max or t.cap, rows, q, o, ws, window=window, sinks=sinks, count=None if counts is None else i32(counts))
    return q, o


def check(t, q, o, rows, counts, window, sinks, layer0=0, left=9.0, faults=0):
    lens = t.c.len.tolist()
    for l in range(q.shape[0]):
        for b, n in enumerate(lens):
            m = min(rows, n) if counts is None else counts[b]
            k, v = t.values(layer0 + l, b)
            pos = np.arange(t.cap) if t.c.pos is None else t.c.pos[b].cpu().numpy()
            x = q[l, b].double().cpu().numpy()[:, :m]
            got = o[l, b].double().cpu().numpy()
            assert (got[:, m:] == left).all(), (l, b)
            want, size, av = reference(x, k, v, seen_of(pos, n, m, window, sinks))
            err = np.abs(got[:, :m] - want)
            lim = limits(t, want, size, av, n, rows)
            assert (err <= lim + 1e-37).all(), (l, b, n, m, err.max(), (err / (lim + 1e-37)).max())
    assert B.faults(t.wws, clear=True) == faults


def cache(lens, rows, places="rows", **kw):
    """places: the rows' numbers (no positions kept), the same kept, or distinct positions in any order, the newest rows' the highest or not."""
    t = Cache(lens, **kw).fill()
    t.wws = B.q4_window_workspace(t.shape, t.cap, rows, t.layers)
    if places == "rows":
        t.c.pos = None
    elif places == "ordered":
        t.c.pos.copy_(torch.arange(t.cap, dtype=torch.int32).expand(len(lens), t.cap))
    elif places == "evicted":  # in some order with gaps; the newest rows behind
        for b, n in enumerate(lens):
            old = max(0, n - rows)
            p = torch.randperm(3 * t.cap, generator=gen(b))[: old].sort().values
            swap = torch.randperm(old, generator=gen(b + 50))[: old // 4]
            p[swap] = p[swap.flip(0)]
            t.c.pos[b, :old] = p.to(torch.int32)
            t.c.pos[b, old:] = torch.arange(3 * t.cap, 4 * t.cap - old, dtype=torch.int32)
    return t  # ("any": Cache's random order)


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("places", ["rows", "any"])
def test_every_group(hq, hkv, d, dtype, places):
    lens = [33, 0, 1, 150, 70]
    for rows, counts, window, sinks in ((1, [1, 0, 1, 1, 1], 20, 3), (41, [33, 0, 1, 41, 7], 24, 5), (41, None, 0, 0)):
        t = cache(lens, rows, places, layers=2, hq=hq, hkv=hkv, d=d, dtype=dtype)
        q, o = run(t, rows, counts, window, sinks)
        check(t, q, o, rows, counts, window, sinks)


@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("lens", [[1], [15, 16, 17], [31, 32, 33, 63, 64, 65], [127, 128, 129], [255, 257, 511, 513], [1000, 3, 2049]])
@pytest.mark.parametrize("places", ["rows", "evicted"])
def test_lengths(page_rows, lens, places):
    for rows, window, sinks in ((1, 100, 4), (1, 0, 0), (9, 31, 17)):
        t = cache(lens, rows, places, page_rows=page_rows, hq=8, hkv=2)
        q, o = run(t, rows, None, window, sinks, n_max=max(lens))
        check(t, q, o, rows, None, window, sinks)


@pytest.mark.parametrize("places", ["rows", "ordered", "evicted", "any"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 5), (1, 0), (1, 1), (2, 64), (31, 0), (32, 1), (33, 33), (500, 0), (2 ** 31 - 1, 0), (7, 2 ** 31 - 1), (3, 200)])
def test_windows(places, window, sinks):
    """Windows that end in every place of a tile; sinks inside the window; a query sees itself in the smallest one."""
    rows, lens, counts = 40, [300, 40, 100], [40, 40, 3]
    t = cache(lens, rows, places, hq=4, hkv=2, page_rows=32)
    q, o = run(t, rows, counts, window, sinks)
    check(t, q, o, rows, counts, window, sinks)
    q, o = run(t, 1, None, window, sinks)
    check(t, q, o, 1, None, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("places", ["rows", "ordered", "evicted"])
def test_long_sequences(dtype, places):
    """Thousands of rows, divided among workgroups; few of them in the window."""
    for rows, window, sinks in ((1, 0, 0), (1, 700, 40), (1, 5, 0), (70, 1000, 3), (70, 0, 0)):
        t = cache([9001, 400, 5000], rows, places, page_rows=64, hq=4, hkv=1, dtype=dtype)
        q, o = run(t, rows, None, window, sinks)
        check(t, q, o, rows, None, window, sinks)


@pytest.mark.parametrize("places", ["rows", "ordered", "any"])
def test_more_rows_than_a_run_of_marks(places):
    """Past 131,072 rows a wave's marks are taken in several runs."""
    n = 141_000
    t = cache([n], 3, places, page_rows=256, hq=2, hkv=1, d=64)
    for rows, window, sinks in ((1, 0, 0), (1, 40_000, 100), (3, 300, 5), (3, 0, 0)):
        q, o = run(t, rows, None, window, sinks)
        check(t, q, o, rows, None, window, sinks)


def test_many_blocks():
    """More blocks of queries than workgroups are wanted: each takes all of its rows."""
    t = cache([600, 513, 700, 1], 512, "rows", layers=2, hq=16, hkv=4, page_rows=64)
    counts = [512, 511, 300, 1]
    q, o = run(t, 512, counts, 128, 4)
    check(t, q, o, 512, counts, 128, 4)


@pytest.mark.parametrize("rows", [1, 6])
def test_strides(rows):
    """Queries and outputs in other orders; one query for all heads, slots and rows."""
    t = cache([50, 40, 33], rows, "rows", layers=2, hq=6, hkv=2)
    shape = (2, 3, 6, rows, 128)
    base = torch.randn(3, rows, 6, 2, 128, generator=gen(5)).bfloat16().cuda()
    q = base.permute(3, 0, 2, 1, 4)
    o = torch.full((6, 2, rows, 3, 160), 9.0, dtype=torch.bfloat16, device="cuda")[..., :128].permute(1, 3, 0, 2, 4)
    assert q.shape == shape and o.shape == shape
    B.kv_q4_attend_window(t.c, 0, 2, t.cap, rows, q, o, t.wws, window=16, sinks=2)
    check(t, q, o, rows, None, 16, 2)
    one = torch.randn(1, 1, 1, 1, 128, generator=gen(6)).bfloat16().cuda().expand(shape)
    B.kv_q4_attend_window(t.c, 0, 2, t.cap, rows, one, o, t.wws, window=16, sinks=2)
    check(t, one, o, rows, None, 16, 2)


@pytest.mark.parametrize("places", ["rows", "any"])
def test_more_queries_than_rows(places):
    """A call may have room for more queries than a slot can have rows."""
    t = cache([20, 0, 33], 300, places, hq=4, hkv=2)
    for counts in (None, [20, 0, 7]):
        q, o = run(t, 300, counts, 9, 2)
        check(t, q, o, 300, counts, 9, 2)


def test_layers():
    t = cache([100, 7], 5, "rows", layers=4, hq=4, hkv=2)
    q, o = run(t, 5, None, 20, 1, layers=2, layer0=1)
    check(t, q, o, 5, None, 20, 1, layer0=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 8])
@pytest.mark.parametrize("places", ["rows", "ordered"])
def test_masked_rows_that_are_not_numbers(dtype, rows, places):
    """NaN keys and values reach the queries that see their rows, values only their block of 32 elements, and no other query."""
    t = cache([80, 80], rows, places, hq=4, hkv=2, dtype=dtype)
    k, v = (torch.randn(1, 2, 2, 80, 128, generator=gen(s)).to(DT[dtype]) for s in (1, 2))
    k[0, 0, :, 75, 3] = float("inf")   # row 75: keys
    v[0, 0, 1, 30, 40] = float("nan")  # row 30, KV head 1: values of elements 32 .. 63
    v[0, 1, :, 79, 100] = float("-inf")  # the newest row of slot 1: elements 96 .. 127
    B.kv_q4_store(t.c, 0, 1, 80, k.cuda(), v.cuda(), t.ws)
    window = 4 if rows == 1 else 20
    q, o = run(t, rows, None, window, 31 if rows > 1 else 0)
    o = torch.isnan(o[0].float()).cpu()  # [slot][head][row][d]
    want = torch.zeros_like(o)
    for r in range(rows):
        at = 80 - rows + r
        want[0, :, r] = 75 <= at < 75 + window
        if rows > 1:
            want[0, 2:, r, 32:64] = True
    want[1, :, rows - 1, 96:] = True
    assert torch.equal(o, want)
    # and what is not NaN is as it is without those rows
    B.kv_q4_store(t.c, 0, 1, 80, torch.nan_to_num(k, nan=0.0, posinf=0.0).cuda(), torch.nan_to_num(v, nan=0.0, neginf=0.0).cuda(), t.ws)
    q2, o2 = run(t, rows, None, window, 31 if rows > 1 else 0)
    check(t, q2, o2, rows, None, window, 31 if rows > 1 else 0)


def test_queries_that_are_not_numbers():
    """Only their own outputs are."""
    t = cache([64], 8, "rows", hq=4, hkv=1)
    q = torch.randn(1, 1, 4, 8, 128, generator=gen(1)).bfloat16()
    q[0, 0, 2, 3, 5], q[0, 0, 1, 7, 0] = float("nan"), float("inf")
    o = torch.full_like(q, 9.0).cuda()
    B.kv_q4_attend_window(t.c, 0, 1, t.cap, 8, q.cuda(), o, t.wws)
    bad = torch.isnan(o[0, 0].float()).all(-1).cpu()
    want = torch.zeros(4, 8, dtype=torch.bool)
    want[2, 3] = want[1, 7] = True
    assert torch.equal(bad, want) and torch.isfinite(o[0, 0].float().cpu()[~want]).all()


def test_positions_at_the_ends_of_their_type():
    t = cache([40], 2, "any", hq=4, hkv=2)
    p = torch.arange(2 ** 31 - 40, 2 ** 31, dtype=torch.int64).to(torch.int32)
    p[:3] = torch.tensor([0, 1, -2 ** 31])
    t.c.pos[0, :40] = p
    for window, sinks in ((5, 1), (2 ** 31 - 1, 0), (0, 0), (1, 2 ** 31 - 1)):
        q, o = run(t, 2, None, window, sinks)
        check(t, q, o, 2, None, window, sinks)


@pytest.mark.parametrize("rows", [1, 5])
def test_slots_that_cannot_be(rows):
    """Lengths and counts out of range: zeros for all of the slot's queries; pages that do not exist: their rows take no part."""
    t = cache([30, 30, 30, 30, 48], rows, "rows", hq=4, hkv=2)
    counts = [1, -1, rows + 1, 1, 1]
    t.c.len.copy_(i32([30, 30, 30, t.cap + 1, 48]))
    t.c.table[4, 1] = t.shape.n_pages + 7  # rows 16 .. 31
    q, o = run(t, rows, counts, 0, 0)
    assert (o[:, 1:4] == 0).all()
    k, v = t.values(0, 0)
    for b, use in ((0, np.ones(30, dtype=bool)), (4, np.r_[np.ones(16, dtype=bool), np.zeros(16, dtype=bool), np.ones(16, dtype=bool)])):
        t.c.table[4, 1] = 0
        k, v = t.values(0, b)
        want, size, av = reference(q[0, b].double().cpu().numpy()[:, :1], k, v, use[None])
        assert (np.abs(o[0, b, :, :1].double().cpu().numpy() - want) <= limits(t, want, size, av, len(use), rows)).all()
        assert (o[0, b, :, 1:] == 9.0).all()
    assert B.faults(t.wws, clear=True) == B.KV_FAULT_CACHE
    t.c.len.copy_(i32([2, -5, 0, 1, 0]))
    q, o = run(t, rows, None, 0, 0)  # without counts: as many as there are
    assert (o[:, 1] == 0).all() and (o[:, 2] == 9.0).all() and (o[:, 4] == 9.0).all() and (o[0, 0, :, 2:] == 9.0).all()
    assert B.faults(t.wws, clear=True) == B.KV_FAULT_CACHE
    if rows > 1:  # a count above the length
        t.c.len.copy_(i32([2, 2, 2, 2, 2]))
        q, o = run(t, rows, [3, 2, 2, 2, 2], 0, 0)
        assert (o[:, 0] == 0).all() and (o[0, 1, :, 2:] == 9.0).all() and B.faults(t.wws, clear=True) == B.KV_FAULT_CACHE


def test_all_rows_of_pages_that_do_not_exist():
    """Queries that see nothing: zeros."""
    t = cache([16], 2, "rows", hq=4, hkv=2)
    t.c.table[0, 0] = -1
    q, o = run(t, 2, None, 4, 0)
    assert (o == 0).all() and B.faults(t.wws, clear=True) == B.KV_FAULT_CACHE


def test_as_the_decode_attention():
    """One query without a window, and positions that do not matter: kv_q4_attend's outputs, but for the order of sums."""
    t = cache([700, 33, 0, 256], 1, "rows", layers=3, hq=8, hkv=2)
    q = torch.randn(3, 4, 8, 128, generator=gen(3)).bfloat16().cuda()
    o, o2 = torch.zeros_like(q), torch.zeros_like(q)
    B.kv_q4_attend(t.c, 0, 3, t.cap, q, o, t.ws)
    B.kv_q4_attend_window(t.c, 0, 3, t.cap, 1, q[:, :, :, None], o2[:, :, :, None], t.wws)
    assert (o.float() - o2.float()).abs().max() <= 2.0 ** -7 * o.float().abs().max()
    assert (o2[:, 2] == 0).all()


def test_workspace_serves_smaller_calls():
    t = cache([1500, 30], 40, "evicted", layers=5, hq=4, hkv=2, page_rows=64)
    ws = B.q4_window_workspace(t.shape, 1500, 40, 5)
    guard = torch.full((ws.numel() + 4096,), 77, dtype=torch.uint8, device="cuda")
    guard[:256] = 0
    for layers in (1, 2, 5):
        for rows in (1, 2, 7, 40):
            for n in (1500, 1501 - 256, 30):
                t.c.len.copy_(i32([min(n, 1500), 30]))
                for window in (0, 64):
                    q, o = run(t, rows, None, window, 2, layers=layers, n_max=n, ws=guard[: ws.numel()])
                    t.wws = guard[: ws.numel()]
                    if layers == 1:
                        check(t, q, o, rows, None, window, 2)
    assert (guard[ws.numel():] == 77).all()


def test_captured_and_replayed():
    """A captured call replays with other lengths, counts, positions and queries; eager calls on another stream between."""
    t = cache([300, 200], 20, "evicted", layers=2, hq=8, hkv=2, page_rows=32)
    other = cache([90], 4, "rows", hq=4, hkv=2)
    q = torch.randn(2, 2, 8, 20, 128, generator=gen(3)).bfloat16().cuda()
    o, count = torch.full_like(q, 9.0), i32([20, 20])

    def call():
        B.kv_q4_attend_window(t.c, 0, 2, t.cap, 20, q, o, t.wws, window=50, sinks=3, count=count)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i, (n, c) in enumerate((([300, 200], [20, 1]), ([37, 199], [0, 20]), ([1, 200], [1, 7]))):
        t.c.len.copy_(i32(n))
        count.copy_(i32(c))
        t.c.pos.copy_(torch.stack([torch.randperm(t.cap, generator=gen(20 + i)) for _ in n]).to(torch.int32))
        q.copy_(torch.randn(q.shape, generator=gen(40 + i)))
        o.fill_(9.0)
        graph.replay()
        with torch.cuda.stream(side):
            q2, o2 = run(other, 4, None, 10, 1)
        check(t, q, o, 20, c, 50, 3)
        side.synchronize()
        check(other, q2, o2, 4, None, 10, 1)


# ---- blocks of four column tiles: bf16 calls whose n_max and queries allow for work for the whole GPU --------------------------------

def roomy(lens, rows, places, page_rows=16, **kw):
    """A cache whose slots could hold 131,072 rows each."""
    return cache(lens, rows, places, page_rows=page_rows, max_pages=131072 // page_rows, **kw)


@pytest.mark.parametrize("hq,hkv,d,page_rows", [(8, 8, 128, 16), (28, 4, 128, 32), (16, 4, 64, 16), (16, 1, 128, 256), (6, 2, 64, 64), (40, 8, 128, 128)])
@pytest.mark.parametrize("places", ["rows", "ordered", "evicted", "any"])
def test_long_blocks(hq, hkv, d, page_rows, places):
    lens = [700, 0, 41, 1, 333]
    for rows, counts, window, sinks in ((70, None, 0, 0), (70, [70, 0, 41, 1, 7], 90_000, 3000), (130, [130, 0, 3, 0, 129], 0, 0)):
        t = roomy(lens, rows, places, page_rows, layers=2, hq=hq, hkv=hkv, d=d)
        q, o = run(t, rows, counts, window, sinks)
        check(t, q, o, rows, counts, window, sinks)


@pytest.mark.parametrize("places", ["rows", "ordered", "any"])
@pytest.mark.parametrize("window,sinks", [(300, 0), (303, 17), (331, 64)])
def test_long_blocks_in_windows(window, sinks, places):
    """Windows that end in several places of a tile, of so many slots and layers that they are worth four column tiles."""
    lens, rows = [350, 401, 70, 290] * 4, 70
    t = cache(lens, rows, places, layers=8, hq=32, hkv=8, page_rows=32)
    q, o = run(t, rows, None, window, sinks)
    check(t, q[:1], o[:1], rows, None, window, sinks)
    check(t, q[7:], o[7:], rows, None, window, sinks, layer0=7)


def test_long_sequences_in_long_blocks():
    """Divided among workgroups, many tiles to a wave."""
    for hq, hkv, layers, rows in ((32, 8, 8, 128), (14, 2, 30, 130)):
        t = cache([4100], rows, "rows", layers=layers, hq=hq, hkv=hkv, page_rows=64)
        q, o = run(t, rows, None, 0, 0)
        check(t, q[:1], o[:1], rows, None, 0, 0)
        check(t, q[layers - 1 :], o[layers - 1 :], rows, None, 0, 0, layer0=layers - 1)


@pytest.mark.parametrize("places", ["rows", "ordered"])
@pytest.mark.parametrize("d", [64, 128])
def test_masked_rows_that_are_not_numbers_in_long_blocks(d, places):
    t = roomy([80, 80], 70, places, hq=16, hkv=4, d=d)
    k, v = (torch.randn(1, 2, 4, 80, d, generator=gen(s)).bfloat16() for s in (1, 2))
    k[0, 0, :, 75, 3] = float("inf")
    v[0, 0, 1, 30, 40] = float("nan")
    v[0, 1, :, 79, 10] = float("-inf")
    B.kv_q4_store(t.c, 0, 1, 80, k.cuda(), v.cuda(), t.ws)
    q, o = run(t, 70, None, 0, 0)
    o = torch.isnan(o[0].float()).cpu()
    want = torch.zeros_like(o)
    want[0, :, 65:] = True           # queries at 75 and behind
    want[0, 4:8, 20:, 32:64] = True  # KV head 1, queries at 30 and behind
    want[1, :, 69, :32] = True
    assert torch.equal(o, want)
    B.kv_q4_store(t.c, 0, 1, 80, torch.nan_to_num(k, nan=0.0, posinf=0.0).cuda(), torch.nan_to_num(v, nan=0.0, neginf=0.0).cuda(), t.ws)
    q, o = run(t, 70, None, 0, 0)
    check(t, q, o, 70, None, 0, 0)


def test_slots_that_cannot_be_in_long_blocks():
    t = roomy([90, 90, 90, 90, 96], 70, "rows", hq=16, hkv=4)
    t.c.len.copy_(i32([90, 90, 90, t.cap + 1, 96]))
    t.c.table[4, 1] = t.shape.n_pages + 7  # rows 16 .. 31
    q, o = run(t, 70, [70, -1, 71, 1, 60], 0, 0)
    assert (o[:, 1:4] == 0).all() and B.faults(t.wws, clear=True) == B.KV_FAULT_CACHE
    for b, count, gone in ((0, 70, ()), (4, 60, range(16, 32))):
        t.c.table[4, 1] = 0
        k, v = t.values(0, b)
        n = k.shape[1]
        seen = seen_of(np.arange(n), n, count, 0, 0)
        seen[:, list(gone)] = False
        want, size, av = reference(q[0, b].double().cpu().numpy()[:, :count], k, v, seen)
        assert (np.abs(o[0, b, :, :count].double().cpu().numpy() - want) <= limits(t, want, size, av, n, 70)).all()
        assert (o[0, b, :, count:] == 9.0).all()


def test_long_blocks_captured_and_replayed():
    t = roomy([300, 200], 70, "evicted", layers=2, hq=16, hkv=4)
    q = torch.randn(2, 2, 16, 70, 128, generator=gen(3)).bfloat16().cuda()
    o, count = torch.full_like(q, 9.0), i32([70, 70])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_q4_attend_window(t.c, 0, 2, t.cap, 70, q, o, t.wws, window=100_000, sinks=3, count=count)
    for i, (n, c) in enumerate((([300, 200], [70, 1]), ([77, 199], [0, 70]), ([1, 200], [1, 7]))):
        t.c.len.copy_(i32(n))
        count.copy_(i32(c))
        t.c.pos.copy_(torch.stack([torch.randperm(t.cap, generator=gen(20 + i)) for _ in n]).to(torch.int32))
        o.fill_(9.0)
        graph.replay()
        _ = (t.c.u * 2).sum().item()
        check(t, q, o, 70, c, 100_000, 3)
