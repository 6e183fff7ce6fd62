"""The paged 4-bit cache on the GPU against the plain float64 model (q4_reference.py).

Tolerances.  Stored and loaded rows, tables, counts, positions and moved utilities: equal.  Attention: products of a query
(bf16: exact; f32: 24 bits) and a stored element (2 bits) are exact or rounded once, and d of them are added in 32 bits: a
logit is off by at most (d + 4) 2^-24 sum |q k| / sqrt(d) and by 2^-23 of itself in the scaling by log2(e) / sqrt(d), a
probability by twice the logits' error, plus the sums over n rows and the exponential (n + 64) 2^-24, all relative; in bf16
the products with values take probabilities of 16 bits (2^-15) and the output is rounded (2^-8 of itself)."""
import numpy as np
import pytest
import torch

import q4_reference as R

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2609_03515_amd.binding")
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """A cache whose slots hold the lengths `lens` in scattered pages; everything unused is random bytes or -1."""

    def __init__(self, lens, layers=1, hq=4, hkv=2, d=128, page_rows=16, dtype="bf16", spare=3, max_pages=None, seed=0, n_pages=None):
        self.lens = list(lens)
        pages = [-(-n // page_rows) for n in lens]
        max_pages = max_pages or max(1, max(pages) + 1)
        n_pages = n_pages or sum(pages) + spare
        self.shape = B.make_q4_shape(len(lens), layers, hq, hkv, d, page_rows, n_pages, max_pages, dtype)
        g = gen(seed)
        self.c = B.KvQ4Cache.allocate(self.shape)
        self.cap = max_pages * page_rows
        perm = torch.randperm(n_pages, generator=g)
        table = torch.full((len(lens), max_pages), -1, dtype=torch.int32)
        at = 0
        for b, p in enumerate(pages):
            table[b, :p] = perm[at : at + p]
            at += p
        self.c.table.copy_(table)
        self.c.len.copy_(torch.tensor(lens))
        refs = torch.zeros(n_pages, dtype=torch.int32)
        refs[perm[:at].long()] = 1
        self.c.refs.copy_(refs)
        raw = torch.randint(0, 256, self.c.pool.shape, generator=g, dtype=torch.uint8)
        self.c.pool.copy_(raw)
        self.c.u.copy_(torch.rand(self.c.u.shape, generator=g))
        self.c.pos.copy_(torch.stack([torch.randperm(self.cap, generator=g) for _ in lens]).to(torch.int32))
        self.ws = B.q4_workspace(self.shape, self.cap, layers)
        self.dtype, self.d, self.hkv, self.hq, self.layers = dtype, d, hkv, hq, layers

    def fill(self, seed=1, scale=1.0):
        """Random rows in every slot."""
        rows = max(self.lens)
        if rows == 0:
            return self
        kv = [torch.randn(self.layers, len(self.lens), self.hkv, rows, self.d, generator=gen(seed + i)).mul_(scale).to(DT[self.dtype]).cuda()
              for i in range(2)]
        B.kv_q4_store(self.c, 0, self.layers, rows, *kv, self.ws, count=self.c.len)
        return self

    def faults(self):
        return B.faults(self.ws, clear=True)

    def values(self, layer, b):
        """Keys and values of a slot, float64, from the pool's bytes."""
        pool = R.Pool(self.shape, self.c.pool.cpu().numpy())
        n = int(self.c.len[b])
        pages = self.c.table[b, : -(-n // self.shape.page_rows)].tolist()
        return pool.sequence(layer, pages, n, True), pool.sequence(layer, pages, n, False)


# ---- rows ---------------------------------------------------------------------------------------------------

def special_rows(shape, seed):
    """Rows with what blocks can hold: all zeros, ties, the exponent's border, the smallest and largest numbers."""
    x = torch.randn(shape, generator=gen(seed), dtype=torch.float64)
    flat = x.view(-1, shape[-1])
    flat *= 2.0 ** torch.randint(-12, 12, (flat.shape[0], 1), generator=gen(seed + 1))
    kinds = [lambda r: r.zero_(), lambda r: r.fill_(-0.0), lambda r: r.copy_(torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0] * (len(r) // 8))),
             lambda r: r.fill_(1.75), lambda r: r.fill_(1.7421875), lambda r: r.mul_(2.0 ** -110), lambda r: r.fill_(3.0e38),
             lambda r: r.mul_(2.0 ** 120), lambda r: r.fill_(2.0 ** -130), lambda r: r.fill_(3.38e38)]
    for i in range(flat.shape[0]):
        if i % 3 == 0:
            kinds[i // 3 % len(kinds)](flat[i])
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page_rows,lens,counts", [
    (128, 16, [5, 0, 40], [5, 0, 33]), (64, 16, [1], [1]), (128, 64, [200, 64], [7, 64]), (64, 256, [300, 17, 256], [299, 1, 0])])
def test_store_and_load(d, page_rows, lens, counts, dtype):
    t = Cache(lens, layers=3, d=d, page_rows=page_rows, dtype=dtype)
    rows = max(max(counts), 1) + 2
    # rows, heads and slots in an order other than the cache's; keys and values in different ones
    k = special_rows((2, len(lens), rows, t.hkv, d), 5).to(DT[dtype]).cuda().transpose(2, 3)
    v = special_rows((len(lens), 2, t.hkv, rows, d), 9).to(DT[dtype]).cuda().transpose(0, 1)
    before = t.c.pool.clone()
    B.kv_q4_store(t.c, 1, 2, rows, k, v, t.ws, count=i32(counts))
    after = t.c.pool.clone()
    pool = R.Pool(t.shape, after.cpu().numpy())
    old, new = (x.view(3, -1).cpu() for x in (before, after))
    assert torch.equal(old[0], new[0])  # a layer that is not the call's
    written = np.zeros((2, t.shape.n_pages, page_rows), dtype=bool)
    for b, (n, m) in enumerate(zip(lens, counts)):
        for l in range(2):
            for name, x, first in (("k", k, True), ("v", v, False)):
                want = R.fast_values(x[l, b, :, :m].double().cpu().numpy())
                got = pool.sequence(1 + l, t.c.table[b].tolist()[: -(-n // page_rows)], n, first)[:, n - m :]
                assert np.array_equal(got, want, equal_nan=True), (b, l, name)
                assert np.array_equal(np.signbit(got)[got == got], np.signbit(want)[got == got])
        for i in range(n - m, n):
            written[:, int(t.c.table[b, i // page_rows]), i % page_rows] = True
    # nothing else changed: rows that were not stored keep their bytes
    a, c = (R.Pool(t.shape, x.cpu().numpy()).rec[1:] for x in (before, after))
    widths = [d // 2, d // 32] * 2
    at = 0
    for w in widths:
        pa, pc = (x[..., at : at + page_rows * w].reshape(2, t.shape.n_pages, t.hkv, page_rows, w) for x in (a, c))
        same = (pa == pc).all(-1).all(2)
        assert same[~written].all()
        at += page_rows * w
    # and back, into rows that are left alone beyond the counts
    k2, v2 = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    B.kv_q4_load(t.c, 1, 2, rows, k2, v2, t.ws, count=i32(counts))
    for b, m in enumerate(counts):
        for x, y in ((k, k2), (v, v2)):
            assert np.array_equal(y[:, b, :, :m].double().cpu().numpy(), R.fast_values(x[:, b, :, :m].double().cpu().numpy()), equal_nan=True)
            assert (y[:, b, :, m:] == 3.0).all()
    assert t.faults() == 0


def test_store_against_the_searching_quantiser():
    """One block of each kind through the model that searches exponents and codes."""
    t = Cache([32], d=64, dtype="f32", hkv=1, hq=1)
    x = special_rows((1, 1, 1, 32, 64), 3).float()
    B.kv_q4_store(t.c, 0, 1, 32, x.cuda(), x.cuda(), t.ws)
    k, _ = t.values(0, 0)
    assert np.array_equal(k[0], R.values(*R.quantise(x[0, 0, 0].double().numpy())), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_that_are_not_finite(dtype):
    t = Cache([6], dtype=dtype)
    x = torch.randn(1, 1, 2, 6, 128, generator=gen(2)).to(DT[dtype])
    x[0, 0, 0, 1, 33], x[0, 0, 1, 4, 127], x[0, 0, 1, 5, 0] = float("nan"), float("inf"), float("-inf")
    B.kv_q4_store(t.c, 0, 1, 6, x.cuda(), x.cuda(), t.ws)
    y = torch.zeros_like(x).cuda()
    B.kv_q4_load(t.c, 0, 1, 6, y, y.clone(), t.ws)
    bad = torch.zeros(1, 1, 2, 6, 4, dtype=torch.bool)
    bad[0, 0, 0, 1, 1] = bad[0, 0, 1, 4, 3] = bad[0, 0, 1, 5, 0] = True
    bad = bad.repeat_interleave(32, -1)
    y = y.cpu()
    assert torch.isnan(y[bad]).all() and not torch.isnan(y[~bad]).any()
    want = R.fast_values(torch.where(bad, torch.zeros(()), x.float()).double().numpy())
    assert np.array_equal(y[~bad].double().numpy(), want[~bad.numpy()])


def test_rows_that_are_not_there():
    """Rows outside the slot, in shared pages and in pages that do not exist are not stored and read as zeros; the others are."""
    t = Cache([20, 40, 16], page_rows=16)
    k = torch.randn(1, 3, 2, 4, 128, generator=gen(1)).bfloat16().cuda()
    t.c.refs[t.c.table[2, 0].long()] = 2
    before = t.c.pool.clone()
    table = t.c.table.clone()
    t.c.table[1, 2] = t.shape.n_pages  # rows 32 .. 39 of slot 1
    B.kv_q4_store(t.c, 0, 1, 4, k, k, t.ws, first=i32([18, 30, 3]))
    assert t.faults() == B.KV_FAULT_CACHE | B.KV_FAULT_SHARED_PAGE
    y = torch.full_like(k, 7.0)
    B.kv_q4_load(t.c, 0, 1, 4, y, y.clone(), t.ws, first=i32([18, 30, -2]))
    assert t.faults() == B.KV_FAULT_CACHE
    want = torch.from_numpy(R.fast_values(k.double().cpu().numpy())).bfloat16().cuda()
    assert torch.equal(y[:, 0, :, :2], want[:, 0, :, :2]) and (y[:, 0, :, 2:] == 0).all()
    assert torch.equal(y[:, 1, :, :2], want[:, 1, :, :2]) and (y[:, 1, :, 2:] == 0).all()
    assert (y[:, 2, :, :2] == 0).all()
    t.c.table.copy_(table)
    own = t.c.pool.view(t.shape.n_pages, -1)
    assert torch.equal(own[table[2, 0].long()], before.view(t.shape.n_pages, -1)[table[2, 0].long()])


# ---- attention ----------------------------------------------------------------------------------------------

def check_attend(t, q, o, cur_pos=None, bias=0.0, window=0, s_out=None, layer0=0, faults=0, lens=None):
    """o (and s_out) of every layer and slot against the model; returns the scores in float64."""
    scores = np.zeros((q.shape[0], len(t.lens), t.cap))
    for l in range(q.shape[0]):
        for b in range(len(t.lens)):
            k, v = t.values(layer0 + l, b)
            n = k.shape[1]
            add = None
            if bias and window:
                add = bias * (t.c.pos[b, :n].cpu().numpy() >= int(cur_pos[b]) - (window - 1))
            want, a, size, av = R.attend(q[l, b].double().cpu().numpy(), k, v, add)
            got = o[l, b].double().cpu().numpy()
            rel = 2 * ((t.d + 4) * 2.0 ** -24 * size + 2.0 ** -22 * (size + abs(bias))) + (n + 64) * 2.0 ** -24
            if t.dtype == "bf16":
                lim = 2.0 ** -8 * np.abs(want) + (rel + 2.0 ** -15) * av * 1.01
            else:
                lim = (rel + 2.0 ** -23) * av
            assert (np.abs(got - want) <= lim + 1e-37).all(), (l, b, np.abs(got - want).max(), lim.min())
            if n:
                scores[l, b, :n] = a.mean(0)
            if s_out is not None:
                s = s_out[l, b].double().cpu().numpy()
                assert (np.abs(s[:n] - scores[l, b, :n]) <= (rel + t.hq * 2.0 ** -24) * scores[l, b, :n] + 1e-37).all(), (l, b)
                assert (s[n:] == 0).all()
    assert t.faults() == faults
    return scores


HEADS = [(4, 4), (4, 2), (6, 2), (8, 2), (10, 2), (12, 2), (7, 1), (8, 1), (9, 1), (16, 1)]


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
def test_attention_of_every_group(hq, hkv, d, dtype):
    t = Cache([33, 0, 1, 150], layers=2, hq=hq, hkv=hkv, d=d, dtype=dtype).fill()
    q = torch.randn(2, 4, hq, d, generator=gen(7)).to(DT[dtype]).cuda()
    o = torch.full_like(q, 9.0)
    s = torch.full((2, 4, t.cap), 9.0, device="cuda")
    B.kv_q4_attend(t.c, 0, 2, t.cap, q, o, t.ws, s_out=s)
    check_attend(t, q, o, s_out=s)
    assert (o[:, 1] == 0).all()
    o2 = torch.full_like(q, 9.0)
    B.kv_q4_attend(t.c, 0, 2, t.cap, q, o2, t.ws)  # without the scores
    check_attend(t, q, o2)


@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("lens", [[1], [15, 16, 17], [31, 32, 33, 63, 64, 65], [127, 128, 129], [255, 257, 511, 513], [1000, 3, 2049]])
def test_attention_lengths(page_rows, lens):
    t = Cache(lens, page_rows=page_rows, hq=8, hkv=2).fill()
    q = torch.randn(1, len(lens), 8, 128, generator=gen(3)).bfloat16().cuda()
    o = torch.empty_like(q)
    n_max = max(lens)
    s = torch.full((1, len(lens), n_max), 9.0, device="cuda")
    B.kv_q4_attend(t.c, 0, 1, n_max, q, o, t.ws, s_out=s)
    check_attend(t, q, o, s_out=s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_a_long_sequence(dtype):
    """Thousands of rows: the call is cut into chunks; one slot is much shorter than the others."""
    t = Cache([9001, 40, 5000], page_rows=64, hq=4, hkv=1, dtype=dtype).fill()
    q = (3 * torch.randn(1, 3, 4, 128, generator=gen(3))).to(DT[dtype]).cuda()
    o = torch.empty_like(q)
    s = torch.full((1, 3, t.cap), 9.0, device="cuda")
    B.kv_q4_attend(t.c, 0, 1, t.cap, q, o, t.ws, s_out=s)
    check_attend(t, q, o, s_out=s)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 8, 64, "bf16"), (32, 8, 128, "bf16"), (24, 8, 128, "f32"), (56, 8, 64, "f32"),
                                            (56, 8, 128, "bf16"), (128, 8, 128, "bf16")])
def test_attention_of_many_slabs(hq, hkv, d, dtype):
    """As many slabs as two for every CU: with scores their logits stay in the workgroup; without, a workgroup has a whole slab.
    Lengths end in every place of a tile's order of rows."""
    lens = [1, 2, 5, 18, 31, 33, 70, 0, 300, 16, 47, 8]
    t = Cache(lens, layers=6, hq=hq, hkv=hkv, d=d, dtype=dtype).fill()
    q = torch.randn(6, 12, hq, d, generator=gen(3)).to(DT[dtype]).cuda()
    cur = i32([t.cap - 1] * 12)
    o, s = torch.full_like(q, 9.0), torch.full((6, 12, 301), 9.0, device="cuda")
    out = torch.full_like(t.c.u, 5.0)
    B.kv_q4_attend(t.c, 0, 6, 301, q, o, t.ws, cur_pos=cur, recency_bias=-0.5, recency_window=100, s_out=s, alpha=0.8,
                   u_prior=t.c.u, u_out=out)
    scores = check_attend(t, q, o, cur, -0.5, 100, s)
    for b, n in enumerate(lens):
        want = t.c.u[b, :n].double().cpu().numpy()
        for l in range(6):
            want = 0.8 * want + 0.2 * scores[l, b, :n]
        lim = 24 * 2.0 ** -24 * want + 2.0 ** -12 * (scores[:, b, :n].sum(0) * 0.2)
        assert (np.abs(out[b, :n].double().cpu().numpy() - want) <= lim).all() and (out[b, n:] == 5.0).all()
    o2 = torch.full_like(q, 9.0)
    B.kv_q4_attend(t.c, 0, 6, 301, q, o2, t.ws, cur_pos=cur, recency_bias=-0.5, recency_window=100)
    check_attend(t, q, o2, cur, -0.5, 100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_in_a_few_chunks(dtype):
    """A hundred slabs of a thousand rows: each in a few chunks, some of which short sequences lack."""
    lens = [1000, 255, 256, 257, 513, 999, 1, 0, 770, 1000, 64, 300, 800]
    t = Cache(lens, layers=2, hq=8, hkv=4, dtype=dtype, page_rows=32).fill()
    q = torch.randn(2, 13, 8, 128, generator=gen(3)).to(DT[dtype]).cuda()
    o, s = torch.full_like(q, 9.0), torch.full((2, 13, 1000), 9.0, device="cuda")
    B.kv_q4_attend(t.c, 0, 2, 1000, q, o, t.ws, s_out=s)
    check_attend(t, q, o, s_out=s)
    B.kv_q4_attend(t.c, 0, 2, 1000, q, o.fill_(9.0), t.ws)
    check_attend(t, q, o)


def test_one_long_sequence_among_many():
    """512 slabs would take a chunk each; no chunk is longer than 8,192 rows."""
    lens = [9000] + [40] * 63
    t = Cache(lens, layers=1, hq=8, hkv=8, d=64, page_rows=256, n_pages=120).fill()
    q = torch.randn(1, 64, 8, 64, generator=gen(3)).bfloat16().cuda()
    o = torch.full_like(q, 9.0)
    B.kv_q4_attend(t.c, 0, 1, 9000, q, o, t.ws)
    check_attend(t, q, o)


def test_scores_with_room_for_many_rows():
    """A call whose n_max, over all slots, is 2^28 rows, 16 waves for 64 of them: the scores of short slots as with a small n_max."""
    n_max, lens = 1 << 22, [5 + 3 * b for b in range(64)]
    small = Cache(lens, hq=16, hkv=16, d=64, page_rows=256, max_pages=1).fill()
    s = B.make_q4_shape(64, 1, 16, 16, 64, 256, small.shape.n_pages, n_max // 256, "bf16")
    table = torch.full((64, n_max // 256), -1, dtype=torch.int32, device="cuda")
    table[:, :1] = small.c.table
    c = B.KvQ4Cache(s, small.c.pool, table, small.c.len, small.c.refs)
    q = torch.randn(1, 64, 16, 64, generator=gen(9)).to(torch.bfloat16).cuda()
    o, want_o = torch.empty_like(q), torch.empty_like(q)
    scores = torch.full((1, 64, n_max), 7.0, device="cuda")
    want = torch.empty(1, 64, 256, device="cuda")
    B.kv_q4_attend(small.c, 0, 1, 256, q, want_o, small.ws, s_out=want)
    ws = B.q4_workspace(s, n_max, 1)
    B.kv_q4_attend(c, 0, 1, n_max, q, o, ws, s_out=scores)
    assert torch.equal(scores[:, :, :256], want) and torch.equal(o, want_o)
    assert not scores[:, :, 256:].any() and B.faults(ws) == 0


def test_workspace_serves_smaller_calls():
    """A workspace for n_max rows and all layers takes every call on fewer of either, whatever way those are divided."""
    t = Cache([1500, 3], layers=5, hq=4, hkv=2, page_rows=64).fill()
    ws = B.q4_workspace(t.shape, 1500, 5)
    q = torch.randn(5, 2, 4, 128, generator=gen(3)).bfloat16().cuda()
    o = torch.empty_like(q)
    s = torch.empty(5 * 2 * 1500, device="cuda")
    ref = torch.empty_like(q)
    B.kv_q4_attend(t.c, 0, 5, 1500, q, ref, ws)
    for n in (1500, 1499, 1281, 1280, 1025, 1024, 513, 512, 300, 256, 255, 1):
        t.c.len.copy_(torch.tensor([min(n, 1500), min(n, 3)]))
        for layers in (1, 2, 3, 4, 5):
            B.kv_q4_attend(t.c, 5 - layers, layers, n, q, o, ws, s_out=s)
    B.kv_q4_evict(t.c, 1, i32([5, 5]), ws)
    B.kv_q4_reserve(t.c, i32([1, 1]), None, ws)
    assert B.faults(ws) == 0


def test_cache_without_utilities():
    """u and pos are optional: pages, rows and attention without them."""
    t = Cache([20, 0, 33], layers=2, d=64)
    c = B.KvQ4Cache(t.shape, t.c.pool, t.c.table, t.c.len, t.c.refs)
    t.c = c
    t.fill()
    B.kv_q4_fork(c, i32([0]), i32([1]), t.ws)
    keep = torch.ones(3, t.cap, dtype=torch.uint8)
    keep[0, 3] = keep[1, 19] = keep[2, ::2] = 0
    before = [[t.values(l, b) for b in range(3)] for l in range(2)]
    B.kv_q4_compact(c, t.cap, keep.cuda(), t.ws)
    assert c.len.tolist() == [19, 19, 16]
    for l in range(2):
        for b, n in ((0, 19), (1, 19)):
            origin = list(range(n))
            if b == 0:
                origin[3] = 19
            for x, y in zip(before[l][b], t.values(l, b)):
                assert np.array_equal(x[:, origin], y)
        for x, y in zip(before[l][2], t.values(l, 2)):
            # rows 1, 3, ... stay: of the places before 16 the even ones are filled with rows 17, 19, ...
            origin = [i if i % 2 else 17 + i for i in range(16)]
            assert np.array_equal(x[:, origin], y)
    B.kv_q4_reserve(c, i32([1, 0, 2]), None, t.ws, init="mean")
    q = torch.randn(2, 3, 4, 64, generator=gen(3)).bfloat16().cuda()
    o = torch.empty_like(q)
    B.kv_q4_attend(c, 0, 2, t.cap, q, o, t.ws)
    t.lens = c.len.tolist()
    check_attend(t, q, o)


def test_first_calls_inside_a_capture():
    """Kernels that need more LDS than the default limit, met for the first time while a graph is captured."""
    t = Cache([2000] * 64, layers=1, hq=40, hkv=8, d=64, dtype="f32", page_rows=256, n_pages=600).fill()
    q = torch.randn(1, 64, 40, 64, generator=gen(3)).cuda()
    o, s = torch.empty_like(q), torch.empty(1, 64, 1000, device="cuda")
    t.c.len.fill_(1000)
    big = Cache([20000], layers=1, hq=1, hkv=1, d=64, page_rows=256)
    start = snapshot(big.c)
    budget = i32([777])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.kv_q4_attend(t.c, 0, 1, 1000, q, o, t.ws, s_out=s)
        B.kv_q4_evict(big.c, 20000, budget, big.ws)
    for _ in range(3):
        restore(big.c, start)
        o.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        o2, s2 = torch.empty_like(q), torch.empty_like(s)
        B.kv_q4_attend(t.c, 0, 1, 1000, q, o2, t.ws, s_out=s2)
        assert torch.equal(o, o2) and torch.equal(s, s2) and int(big.c.len[0]) == 777
    assert t.faults() == 0 and big.faults() == 0


def test_recency_bias_and_fold():
    """The bias on recent positions, and the fold of two layers at once and of one layer after the other."""
    t = Cache([70, 33, 0], layers=2, hq=8, hkv=2).fill()
    q = torch.randn(2, 3, 8, 128, generator=gen(3)).bfloat16().cuda()
    cur = i32([t.cap - 1, 40, 3])
    o, s = torch.empty_like(q), torch.empty(2, 3, t.cap, device="cuda")
    prior = t.c.u.clone()
    out = torch.full_like(prior, 5.0)
    B.kv_q4_attend(t.c, 0, 2, t.cap, q, o, t.ws, cur_pos=cur, recency_bias=0.75, recency_window=30, s_out=s, alpha=0.9,
                   u_prior=prior, u_out=out)
    scores = check_attend(t, q, o, cur, 0.75, 30, s)
    assert torch.equal(prior, t.c.u)
    for b, n in enumerate(t.lens):
        want = prior[b, :n].double().cpu().numpy()
        for l in range(2):
            want = 0.9 * want + 0.1 * scores[l, b, :n]
        # the scores' error of the attention (under 2^-12 here, times their weight), the coefficients' and three roundings a layer
        lim = 8 * 2.0 ** -24 * want + 2.0 ** -12 * (scores[:, b, :n].sum(0) * 0.1)
        assert (np.abs(out[b, :n].double().cpu().numpy() - want) <= lim).all()
        assert (out[b, n:] == 5.0).all()
    # layer by layer, in place
    for l in range(2):
        B.kv_q4_attend(t.c, l, 1, t.cap, q[l], o[l], t.ws, cur_pos=cur, recency_bias=0.75, recency_window=30, alpha=0.9,
                       u_prior=prior, u_out=prior)
    check_attend(t, q, o, cur, 0.75, 30)
    for b, n in enumerate(t.lens):
        # the same numbers but for the attention's order of sums (a layer's call may cut its rows otherwise)
        assert torch.allclose(prior[b, :n], out[b, :n], rtol=1e-5, atol=0)
        assert torch.equal(prior[b, n:], t.c.u[b, n:])


def test_unused_rows_and_pages_do_not_matter():
    """Bytes behind the last row, in unused pages and in the table behind the sequence change nothing, not even as NaN."""
    t = Cache([37, 5], page_rows=32).fill()
    q = torch.randn(1, 2, 4, 128, generator=gen(3)).bfloat16().cuda()
    o, s = torch.empty_like(q), torch.empty(1, 2, t.cap, device="cuda")
    B.kv_q4_attend(t.c, 0, 1, t.cap, q, o, t.ws, s_out=s)
    kv = [torch.zeros(1, 2, 2, 64, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.kv_q4_load(t.c, 0, 1, 64, *kv, t.ws, first=i32([0, 0]), count=t.c.len)
    for byte in (0, 255):
        t.c.pool.fill_(byte)
        B.kv_q4_store(t.c, 0, 1, 64, *kv, t.ws, first=i32([0, 0]), count=t.c.len)
        t.c.table[0, 2] = -7  # behind the sequence
        t.c.table[1, 1:] = 1 << 30
        o2, s2 = torch.empty_like(q), torch.empty_like(s)
        B.kv_q4_attend(t.c, 0, 1, t.cap, q, o2, t.ws, s_out=s2)
        assert torch.equal(o, o2) and torch.equal(s, s2)
    assert t.faults() == 0


def test_bad_state_is_left_out():
    """A length out of range: zeros; a page that does not exist: its rows take no part."""
    t = Cache([40, 20, 64, 50], page_rows=16).fill()
    q = torch.randn(1, 4, 4, 128, generator=gen(3)).bfloat16().cuda()
    ref = torch.empty_like(q)
    o, s = torch.empty_like(q), torch.empty(1, 4, 48, device="cuda")
    k, v = t.values(0, 3)
    t.c.len[1], t.c.len[2] = -5, 64  # n_max is 48
    t.c.len[3] = 48
    t.c.table[3, 1] = t.shape.n_pages
    B.kv_q4_attend(t.c, 0, 1, 48, q, o, t.ws, s_out=s)
    assert t.faults() == B.KV_FAULT_CACHE
    assert (o[:, 1:3] == 0).all() and (s[:, 1:3] == 0).all() and (s[:, 3, 16:32] == 0).all()
    live = np.r_[0:16, 32:48]
    want, a, _, av = R.attend(q[0, 3].double().cpu().numpy(), k[:, live], v[:, live])
    assert (np.abs(o[0, 3].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * av).all()
    assert np.allclose(s[0, 3, live].double().cpu().numpy(), a.mean(0), rtol=1e-4, atol=0)
    t.c.table[3, :] = -1  # no row left at all
    B.kv_q4_attend(t.c, 0, 1, 48, q, o, t.ws, s_out=s)
    assert (o[:, 3] == 0).all() and (s[:, 3] == 0).all() and t.faults() == B.KV_FAULT_CACHE


def test_rows_that_are_nan():
    """A key or value block that is not finite makes its heads' outputs NaN, as a product with NaN does, and no others."""
    t = Cache([40, 40], hq=8, hkv=4)
    kv = [torch.randn(1, 2, 4, 40, 128, generator=gen(i)).bfloat16() for i in range(2)]
    kv[0][0, 0, 1, 17, 100] = float("inf")
    kv[1][0, 1, 2, 39, 3] = float("nan")
    B.kv_q4_store(t.c, 0, 1, 40, kv[0].cuda(), kv[1].cuda(), t.ws)
    q = torch.randn(1, 2, 8, 128, generator=gen(3)).bfloat16().cuda()
    o = torch.empty_like(q)
    B.kv_q4_attend(t.c, 0, 1, t.cap, q, o, t.ws)
    nan = torch.isnan(o[0]).cpu()
    want = torch.zeros(2, 8, 128, dtype=torch.bool)
    want[0, 2:4] = True            # every output of the two heads of that key's head
    want[1, 4:6, :32] = True       # the columns of the value's block
    assert torch.equal(nan, want)


def test_peaked_and_shifted_logits():
    """One row far above the others, at either end; large equal logits; a growing sequence of maxima."""
    for case in range(4):
        t = Cache([300], hq=4, hkv=1, dtype="f32")
        k = 0.1 * torch.randn(1, 1, 1, 300, 128, generator=gen(1))
        v = torch.randn(1, 1, 1, 300, 128, generator=gen(2))
        q = torch.randn(1, 1, 4, 128, generator=gen(3))
        if case < 2:
            k[0, 0, 0, 299 if case else 0] = 4 * q[0, 0, 0]
        elif case == 2:
            k += 8 * q[0, 0, 0]
        else:
            k += 0.02 * torch.arange(300)[:, None] * q[0, 0, 0]
        B.kv_q4_store(t.c, 0, 1, 300, k.cuda(), v.cuda(), t.ws)
        q, o = q.cuda(), torch.empty(1, 1, 4, 128, device="cuda")
        s = torch.empty(1, 1, t.cap, device="cuda")
        B.kv_q4_attend(t.c, 0, 1, t.cap, q, o, t.ws, s_out=s)
        check_attend(t, q, o, s_out=s)


def test_pages_past_four_gigabytes():
    """Offsets of 33 bits: the pages lie at the end of a pool of 5 GB."""
    rows, n_pages = 256, 5 * 2 ** 30 // (2 * 2 * 256 * 136)
    c = B.KvQ4Cache.allocate(B.make_q4_shape(1, 2, 8, 2, 128, 256, n_pages, 4, "bf16"))
    assert c.pool.numel() > 2 ** 32
    ws = B.q4_workspace(c.shape, 1024, 2)
    c.refs[: n_pages - 3] = 1
    B.kv_q4_reserve(c, i32([600]), i32([0]), ws)
    assert c.table[0, :3].tolist() == [n_pages - 3, n_pages - 2, n_pages - 1] and int(c.len[0]) == 600
    k, v = (torch.randn(2, 1, 2, 600, 128, generator=gen(i)).bfloat16().cuda() for i in range(2))
    B.kv_q4_store(c, 0, 2, 600, k, v, ws)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    B.kv_q4_load(c, 0, 2, 600, k2, v2, ws)
    for x, y in ((k, k2), (v, v2)):
        assert np.array_equal(y.double().cpu().numpy(), R.fast_values(x.double().cpu().numpy()))
    q = torch.randn(2, 1, 8, 128, generator=gen(3)).bfloat16().cuda()
    o = torch.empty_like(q)
    B.kv_q4_attend(c, 0, 2, 600, q, o, ws)
    for l in range(2):
        want, _, _, av = R.attend(q[l, 0].double().cpu().numpy(), k2[l, 0].double().cpu().numpy(), v2[l, 0].double().cpu().numpy())
        assert (np.abs(o[l, 0].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * av).all()
    B.kv_q4_evict(c, 600, i32([100]), ws)
    assert int(c.len[0]) == 100 and c.table[0].tolist() == [n_pages - 3, -1, -1, -1] and B.faults(ws) == 0


# ---- pages --------------------------------------------------------------------------------------------------

class Twin:
    """A cache and the Python model of its pages, driven together.  Stored rows are numbered tokens, recognised by their keys."""

    def __init__(self, batch=4, n_pages=24, max_pages=8, page_rows=16, layers=2, hkv=2, d=64, dtype="bf16"):
        self.shape = B.make_q4_shape(batch, layers, hkv, hkv, d, page_rows, n_pages, max_pages, dtype)
        self.c = B.KvQ4Cache.allocate(self.shape)
        self.c.pool.copy_(torch.randint(0, 256, self.c.pool.shape, generator=gen(0), dtype=torch.uint8))
        self.cap = max_pages * page_rows
        self.ws = B.q4_workspace(self.shape, self.cap, layers)
        self.m = R.Pages(batch, n_pages, max_pages, page_rows)
        self.batch, self.token, self.faults = batch, 0, 0

    def _codes(self, token):
        """A token's row: exact in the format, different for each token, layer and head."""
        s = self.shape
        x = np.zeros((s.layers, s.n_kv_heads, s.head_dim))
        for l in range(s.layers):
            for g in range(s.n_kv_heads):
                bits = (token * 8 + l * 2 + g) * 7 + 1
                x[l, g, :32] = [6.0 if bits >> i & 1 else -6.0 for i in range(32)]
                x[l, g, 32:] = [4.0 if bits >> i % 32 & 1 else -6.0 for i in range(s.head_dim - 32)]
        return x

    def append(self, add, pos, init="zero"):
        granted = torch.full((self.batch,), -1, dtype=torch.int32, device="cuda")
        B.kv_q4_reserve(self.c, i32(add), i32(pos), self.ws, granted=granted, init=init)
        prior = {"zero": lambda u: 0.0, "mean": lambda u: float(np.float32(np.mean(u))) if u else 0.0,
                 "min": lambda u: min(u) if u else 0.0}[init]
        want = self.m.reserve(add, pos, prior)
        assert granted.tolist() == want, (granted.tolist(), want)
        rows = max(max(want), 1)
        x = np.zeros((self.shape.layers, self.batch, self.shape.n_kv_heads, rows, self.shape.head_dim))
        for b, n in enumerate(want):
            for r in range(n):
                self.token += 1
                self.m.store(b, self.m.len[b] - n + r, self.token)
                x[:, b, :, r] = self._codes(self.token)
        k = torch.from_numpy(x).to(self.c.element).cuda()
        B.kv_q4_store(self.c, 0, self.shape.layers, rows, k, -k, self.ws, count=granted)
        return want

    def set_u(self, seed):
        u = torch.rand(self.batch, self.cap, generator=gen(seed))
        u = (u * 8).round() / 8 if seed % 2 else u  # many ties
        for b in range(self.batch):
            for i in range(self.m.len[b]):
                self.m.u[b][i] = float(u[b, i])
            self.c.u[b, : self.m.len[b]] = u[b, : self.m.len[b]].cuda()

    def check(self, faults=0):
        m, c = self.m, self.c
        assert c.len.tolist() == m.len
        assert c.table.tolist() == [t + [-1] * (m.max_pages - len(t)) for t in m.table]
        assert c.refs.tolist() == m.refs
        assert B.faults(self.ws, clear=True) == faults
        u, pos = c.u.cpu(), c.pos.cpu()
        pool = R.Pool(self.shape, c.pool.cpu().numpy())
        for b in range(self.batch):
            assert u[b, : m.len[b]].tolist() == [m.u[b][i] for i in range(m.len[b])], b
            assert pos[b, : m.len[b]].tolist() == [m.pos[b][i] for i in range(m.len[b])], b
            want = np.array([self._codes(t) for t in m.tokens(b)]) if m.len[b] else np.zeros((0,))
            for l in range(self.shape.layers):
                for first, sign in ((True, 1.0), (False, -1.0)):
                    got = pool.sequence(l, m.table[b], m.len[b], first)
                    if m.len[b]:
                        assert np.array_equal(got.transpose(1, 0, 2), sign * want[:, l]), (b, l, first)


def test_reserve_grows_and_runs_out():
    t = Twin(batch=3, n_pages=7, max_pages=4)
    t.append([5, 0, 16], [0, 9, 100])
    t.check()
    t.append([11, 0, 1], [5, 0, 116], "mean")     # up to the page's end; one row into the next
    t.check()
    t.append([1, 33, 0], [16, 0, 0], "min")
    t.check()
    assert t.append([50, 0, 1], [0, 0, 0]) == [0, 0, 1]   # past its capacity
    t.check(B.KV_FAULT_CACHE)
    assert t.append([40, 1, 30], [0, 0, 0]) == [0, 1, 0]  # two pages needed, then none, then one; one is free
    t.check(B.KV_FAULT_NO_PAGES)
    assert t.append([-1, 0, 0], [0, 0, 0]) == [0, 0, 0]
    t.check(B.KV_FAULT_CACHE)


def test_reserve_in_place_of_its_counts():
    """granted may be add itself."""
    t = Twin(batch=2, n_pages=2, max_pages=4)
    add = i32([16, 40])
    B.kv_q4_reserve(t.c, add, None, t.ws, granted=add)
    assert add.tolist() == [16, 0] and t.c.len.tolist() == [16, 0]
    assert B.faults(t.ws, clear=True) == B.KV_FAULT_NO_PAGES


def test_fork_shares_and_copies_on_write():
    t = Twin(batch=5, n_pages=12)
    t.append([20, 0, 0, 16, 0], [0, 0, 0, 50, 0])
    t.set_u(2)
    B.kv_q4_fork(t.c, i32([0, 0, 3]), i32([1, 4, 2]), t.ws)
    t.m.fork([0, 0, 3], [1, 4, 2])
    t.check()
    t.append([1, 0, 1, 0, 0], [20, 0, 16, 0, 0], "mean")  # the partial page is copied; a full one needs none
    t.check()
    t.append([1, 2, 0, 1, 30], [21, 20, 0, 16, 20], "min")
    t.check()
    for slots in ([1, 1], [0, 2, 4], [3]):
        B.kv_q4_free(t.c, i32(slots), t.ws)
        t.m.free(slots)
        t.check()
    assert not t.c.refs.any()


def test_fork_refusals():
    t = Twin(batch=5, n_pages=12)
    t.append([20, 0, 0, 5, 0], [0] * 5)
    # in turn: destination not empty; out of range; a source that is a destination; the same slot; named twice
    for src, dst in (([0], [3]), ([0, 0], [5, -1]), ([0, 1], [1, 2]), ([1], [1]), ([7], [1]), ([0, 3], [1, 1]), ([3, 0], [3, 2])):
        B.kv_q4_fork(t.c, i32(src), i32(dst), t.ws)
        t.m.fork(src, dst)
        t.check(B.KV_FAULT_CACHE)
    B.kv_q4_free(t.c, i32([9, 0, -1]), t.ws)
    t.m.free([0])
    t.check(B.KV_FAULT_CACHE)


@pytest.mark.parametrize("page_rows", [16, 64])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f32")])
def test_evict_and_compact(page_rows, d, dtype):
    t = Twin(batch=4, n_pages=40, max_pages=6, page_rows=page_rows, d=d, dtype=dtype)
    t.append([3 * page_rows + 5, 2 * page_rows, 1, 0], [0, 0, 0, 0])
    for step, budget in enumerate(([100000, page_rows + 3, 1, 4], [2 * page_rows, page_rows + 3, 0, 0], [7, 1, 5, 0], [0, 1, 1, 1])):
        t.set_u(step)
        keep_out = torch.full((4, t.cap), 9, dtype=torch.uint8, device="cuda")
        keep = [t.m.best(b, n) for b, n in enumerate(budget)]
        B.kv_q4_evict(t.c, t.cap, i32(budget), t.ws, keep_out=keep_out)
        lens = list(t.m.len)
        t.m.compact(keep)
        t.check()
        for b, n in enumerate(lens):
            assert keep_out[b, :n].tolist() == [int(x) for x in keep[b]] and (keep_out[b, n:] == 9).all()
        t.append([5, 17, 0, 2], [1000 + 100 * step] * 4, "mean")
        t.check()
    masks = torch.zeros(4, t.cap, dtype=torch.uint8)
    g = gen(5)
    for b in range(4):
        masks[b] = torch.randint(0, 3, (t.cap,), generator=g)  # (any value but 0 keeps)
    B.kv_q4_compact(t.c, t.cap, masks.cuda(), t.ws)
    t.m.compact([masks[b, : t.m.len[b]].tolist() for b in range(4)])
    t.check()


def test_evict_of_shared_pages():
    """Slots that share pages evict each for itself: pages with a hole are replaced, whole ones stay shared."""
    t = Twin(batch=4, n_pages=30, max_pages=6)
    t.append([70, 0, 0, 0], [0] * 4)
    B.kv_q4_fork(t.c, i32([0, 0, 0]), i32([1, 2, 3]), t.ws)
    t.m.fork([0, 0, 0], [1, 2, 3])
    for seed in range(3):
        t.set_u(seed)
        budget = [64 - seed, 50, 33, 100]
        keep = [t.m.best(b, n) for b, n in enumerate(budget)]
        B.kv_q4_evict(t.c, t.cap, i32(budget), t.ws)
        t.m.compact(keep)
        t.check()
        t.append([3, 0, 17, 1], [200 * seed + 100] * 4)
        t.check()


def test_compact_without_enough_pages():
    """Slots whose copies do not fit are left as they were; those before them and those that need none are compacted."""
    t = Twin(batch=4, n_pages=6, max_pages=4)
    t.append([40, 0, 0, 16], [0] * 4)
    B.kv_q4_fork(t.c, i32([0, 0]), i32([1, 2]), t.ws)
    t.m.fork([0, 0], [1, 2])
    t.check()  # two free pages left
    t.set_u(4)
    masks = torch.ones(4, t.cap, dtype=torch.uint8)
    masks[0, 3] = masks[1, 2] = masks[1, 20] = masks[2, 20] = masks[3, 0] = 0  # one page, two pages, one, none
    B.kv_q4_compact(t.c, t.cap, masks.cuda(), t.ws)
    t.m.compact([masks[b, : t.m.len[b]].tolist() for b in range(4)])
    t.check(B.KV_FAULT_NO_PAGES)
    assert t.c.len.tolist() == [39, 40, 40, 15]


def test_evict_of_bad_slots():
    """Longer than n_max, a negative budget, a page that does not exist: left alone, the others evicted."""
    t = Twin(batch=4, n_pages=30, max_pages=6)
    t.append([50, 20, 30, 30], [0] * 4)
    t.set_u(2)
    table = t.c.table.clone()
    t.c.table[2, 1] = 31
    B.kv_q4_evict(t.c, 40, i32([5, -1, 10, 7]), t.ws)
    t.c.table[2, 1] = table[2, 1]
    t.m.compact([[True] * 50, [True] * 20, [True] * 30, t.m.best(3, 7)])
    t.check(B.KV_FAULT_CACHE)


@pytest.mark.parametrize("n,budget", [(5000, 4999), (5000, 4996), (5000, 500), (3000, 1), (20000, 12345), (33000, 32000), (140000, 70001)])
def test_evict_of_long_sequences(n, budget):
    """Utilities that share all but their last bits, ties across the border, and infinities among them."""
    pages = -(-n // 128) + 1
    c = B.KvQ4Cache.allocate(B.make_q4_shape(3, 1, 1, 1, 64, 128, 3 * pages, pages, "bf16"))
    ws = B.q4_workspace(c.shape, n, 1)
    B.kv_q4_reserve(c, i32([n, n, n]), i32([0, 0, 0]), ws)
    u = torch.empty(3, n)
    u[0] = (torch.randint(0, 1 << 12, (n,), generator=gen(1)) + 0x3f800000).to(torch.int32).view(torch.float32)
    u[1] = torch.randint(0, 3, (n,), generator=gen(2)).float()
    u[2] = torch.randn(n, generator=gen(3))
    u[2, 7], u[2, 9], u[2, 11] = float("inf"), float("-inf"), -0.0
    pos = torch.stack([torch.randperm(1 << 20, generator=gen(i))[:n] for i in range(3)]).to(torch.int32)
    c.u[:, :n], c.pos[:, :n] = u.cuda(), pos.cuda()
    keep = torch.zeros(3, pages * 128, dtype=torch.uint8, device="cuda")
    B.kv_q4_evict(c, n, i32([budget] * 3), ws, keep_out=keep)
    for b in range(3):
        order = np.lexsort((pos[b].numpy(), -u[b].double().numpy()))[:budget]
        want = np.zeros(n, dtype=np.uint8)
        want[order] = 1
        assert np.array_equal(keep[b, :n].cpu().numpy(), want), b


@pytest.mark.parametrize("n,budget", [(5, 2), (100, 97), (100, 40), (256, 255), (257, 100), (1024, 1000), (1025, 30), (5000, 4996), (5000, 4000), (32768, 12000),
                                      (33000, 9000), (140000, 139999)])
def test_evict_of_rows_that_tie(n, budget):
    """Rows alike in utility (0 and -0 are) and position, as where a caller sets no positions: exactly `budget` stay, the lower
    rows; positions below 0 are lower than others."""
    pages = -(-n // 128) + 1
    c = B.KvQ4Cache.allocate(B.make_q4_shape(3, 1, 1, 1, 64, 128, 3 * pages, pages, "bf16"))
    ws = B.q4_workspace(c.shape, n, 1)
    B.kv_q4_reserve(c, i32([n, n, n]), None, ws)
    u = torch.tensor([0.0, -0.0, 0.5])[torch.randint(0, 3, (3, n), generator=gen(7))]
    pos = torch.tensor([-(1 << 31), -3, 0, 2, (1 << 31) - 1], dtype=torch.int32)[torch.randint(0, 5, (3, n), generator=gen(8))]
    u[1], pos[1] = 0.25, 0  # (all alike)
    u[2] = 0.0
    c.u[:, :n], c.pos[:, :n] = u.cuda(), pos.cuda()
    keep = torch.zeros(3, pages * 128, dtype=torch.uint8, device="cuda")
    B.kv_q4_evict(c, n, i32([budget] * 3), ws, keep_out=keep)
    assert c.len.tolist() == [budget] * 3
    for b in range(3):
        want = np.zeros(n, dtype=np.uint8)
        want[np.lexsort((np.arange(n), pos[b].numpy(), -u[b].double().numpy()))[:budget]] = 1
        assert np.array_equal(keep[b, :n].cpu().numpy(), want), b
        hole, move = np.nonzero(want[:budget] == 0)[0], budget + np.nonzero(want[budget:])[0]
        origin = np.arange(budget)
        origin[hole] = move
        assert np.array_equal(c.pos[b, :budget].cpu().numpy(), pos[b].numpy()[origin])
    assert c.len.tolist() == [budget] * 3 and B.faults(ws) == 0


@pytest.mark.parametrize("page_rows,steps,kw", [(16, 150, dict(layers=1, hkv=1)), (32, 60, dict(layers=2, hkv=3, d=128, dtype="f32")),
                                                (256, 40, dict(layers=1, hkv=2))])
def test_any_order_of_page_calls(page_rows, steps, kw):
    """Calls drawn at random, checked after each."""
    r = np.random.RandomState(11)
    t = Twin(batch=6, n_pages=26, max_pages=5, page_rows=page_rows, **kw)
    most = 25 * page_rows // 16
    for step in range(steps):
        kind = r.randint(5)
        if kind == 0:
            t.append([int(x) for x in r.randint(0, most, 6) * (r.rand(6) < 0.5)], [10000 * step] * 6, ("mean", "min", "zero")[step % 3])
            B.kv_fault_status(t.ws, None, clear=True)
        elif kind == 1:
            src, dst = [int(x) for x in r.randint(0, 6, 2)], [int(x) for x in r.randint(0, 6, 2)]
            B.kv_q4_fork(t.c, i32(src), i32(dst), t.ws)
            t.m.fork(src, dst)
            B.kv_fault_status(t.ws, None, clear=True)
        elif kind == 2:
            slots = [int(x) for x in r.randint(0, 6, r.randint(1, 3))]
            B.kv_q4_free(t.c, i32(slots), t.ws)
            t.m.free(slots)
        else:
            t.set_u(step)
            budget = [int(x) for x in r.randint(0, 60 * page_rows // 16, 6)]
            keep = [t.m.best(b, n) for b, n in enumerate(budget)]
            B.kv_q4_evict(t.c, t.cap, i32(budget), t.ws)
            t.m.compact(keep)
            B.kv_fault_status(t.ws, None, clear=True)
        t.check()


# ---- together -----------------------------------------------------------------------------------------------

def decode(t, q, k, v, o, add, granted, new_pos, budget):
    """One decode step of every slot as a serving loop makes it: a row, attention layer by layer with the fold, eviction."""
    c, L = t.c, t.layers
    B.kv_q4_reserve(c, add, new_pos, t.ws, granted=granted, init="zero")
    for l in range(L):
        B.kv_q4_store(c, l, 1, 1, k[l : l + 1], v[l : l + 1], t.ws, count=granted)
        B.kv_q4_attend(c, l, 1, t.cap, q[l], o[l], t.ws, cur_pos=new_pos, recency_bias=0.5, recency_window=8, alpha=0.9,
                       u_prior=c.u, u_out=c.u)
    B.kv_q4_evict(c, t.cap, budget, t.ws)


STATE = ("pool", "table", "len", "refs", "u", "pos")


def snapshot(c):
    return {name: getattr(c, name).clone() for name in STATE}


def restore(c, s):
    for name in STATE:
        getattr(c, name).copy_(s[name])


def same(a, b, lens, cap):
    for name in ("table", "len", "refs"):
        assert torch.equal(a[name], b[name]), name
    for i, n in enumerate(lens):
        assert torch.equal(a["u"][i, :n], b["u"][i, :n]) and torch.equal(a["pos"][i, :n], b["pos"][i, :n]), i


def decode_inputs(t, steps, seed):
    b = len(t.lens)
    out = []
    for i in range(steps):
        g = gen(seed + i)
        q = torch.randn(t.layers, b, t.hq, t.d, generator=g).to(DT[t.dtype]).cuda()
        k, v = (torch.randn(t.layers, b, t.hkv, 1, t.d, generator=g).to(DT[t.dtype]).cuda() for _ in range(2))
        out.append((q, k, v))
    return out


def test_decode_loop():
    """Prompts stored, samples forked, decode steps with attention, fold and eviction: after every step the attention matches
    the model on the cache's own values, the fold the scores, and the state what the model does with the cache's utilities."""
    t = Cache([40, 23, 0, 0, 0], layers=2, hq=8, hkv=2, d=64, page_rows=16, max_pages=5, n_pages=30).fill()
    t.c.pos[:] = torch.arange(t.cap, dtype=torch.int32, device="cuda")
    t.lens = [0] * 5
    B.kv_q4_fork(t.c, i32([0, 0, 1]), i32([2, 3, 4]), t.ws)
    budget = i32([30, 100, 40, 41, 12])
    for step, (q, k, v) in enumerate(decode_inputs(t, 6, 100)):
        o = torch.empty_like(q)
        add, granted, new_pos = i32([1, 1, 1, 0, 1]), i32([0] * 5), i32([100 + step] * 5)
        B.kv_q4_reserve(t.c, add, new_pos, t.ws, granted=granted, init="zero")
        assert granted.tolist() == [1, 1, 1, 0, 1]
        B.kv_q4_store(t.c, 0, 2, 1, k, v, t.ws, count=granted)
        newest = [t.values(1, b)[0][:, -1] for b in range(5)]
        for b in (0, 1, 2, 4):
            assert np.array_equal(newest[b], R.fast_values(k[1, b, :, 0].double().cpu().numpy()))
        prior = t.c.u.clone()
        s = torch.empty(2, 5, t.cap, device="cuda")
        B.kv_q4_attend(t.c, 0, 2, t.cap, q, o, t.ws, cur_pos=new_pos, recency_bias=0.5, recency_window=8, s_out=s, alpha=0.9,
                       u_prior=prior, u_out=t.c.u)
        check_attend(t, q, o, new_pos, 0.5, 8, s)
        lens, u, pos = t.c.len.tolist(), t.c.u.cpu(), t.c.pos.cpu()
        rows = [np.concatenate(t.values(0, b), -1).transpose(1, 0, 2) for b in range(5)]
        B.kv_q4_evict(t.c, t.cap, budget, t.ws)
        for b, n in enumerate(lens):
            m = min(int(budget[b]), n)
            order = sorted(range(n), key=lambda i: (-float(u[b, i]), int(pos[b, i])))[:m]
            origin, kept = list(range(m)), set(order)
            for hole, move in zip([i for i in range(m) if i not in kept], sorted(i for i in kept if i >= m)):
                origin[hole] = move
            assert int(t.c.len[b]) == m and t.c.pos[b, :m].tolist() == pos[b, origin].tolist()
            assert t.c.u[b, :m].tolist() == u[b, origin].tolist()
            assert np.array_equal(np.concatenate(t.values(0, b), -1).transpose(1, 0, 2), rows[b][origin]), (step, b)
        refs = torch.zeros(t.shape.n_pages, dtype=torch.int32)
        for p in t.c.table.cpu().flatten().tolist():
            if p >= 0:
                refs[p] += 1
        assert torch.equal(refs, t.c.refs.cpu())


def test_captured_decode_steps():
    """Two decode steps in a graph, replayed between eager work: each replay leaves what the eager calls leave, and follows
    lengths and budgets that change between replays."""
    t = Cache([40, 23, 0, 64], layers=2, hq=8, hkv=2, d=128, page_rows=16, max_pages=6, n_pages=40).fill()
    ins = decode_inputs(t, 2, 50)
    o = [torch.empty_like(q) for q, _, _ in ins]
    add, granted, new_pos, budget = i32([1, 1, 0, 1]), i32([0] * 4), i32([200] * 4), i32([30, 100, 5, 64])

    def steps():
        for (q, k, v), out in zip(ins, o):
            decode(t, q, k, v, out, add, granted, new_pos, budget)

    start = snapshot(t.c)
    steps()
    torch.cuda.synchronize()
    restore(t.c, start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    for rep in range(4):
        if rep == 2:
            budget.copy_(i32([10, 11, 5, 33]))
            add.copy_(i32([1, 0, 1, 1]))
        restore(t.c, start)
        steps()
        want, wo = snapshot(t.c), [x.clone() for x in o]
        restore(t.c, start)
        for x in o:
            x.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = snapshot(t.c)
        same(got, want, want["len"].tolist(), t.cap)
        assert torch.equal(got["pool"], want["pool"])
        for x, y in zip(o, wo):
            assert torch.equal(x, y)
        _ = (t.c.u * 2).sum().item()
    assert t.faults() == 0


def test_side_stream_and_two_caches():
    """Calls on a side stream, and on two caches with workspaces of their own at once, give what they give alone."""
    pair = [Cache([50, 21], layers=2, hq=8, hkv=2, seed=i, page_rows=16, max_pages=6, n_pages=20).fill(seed=3 + i) for i in range(2)]
    ins = [decode_inputs(t, 3, 70 + 10 * i) for i, t in enumerate(pair)]
    add, new_pos, budget = i32([1, 1]), i32([300, 300]), i32([40, 60])
    streams = [torch.cuda.Stream() for _ in pair]
    starts = [snapshot(t.c) for t in pair]
    results = []
    for side in (False, True):
        outs = [[torch.empty_like(q) for q, _, _ in x] for x in ins]
        granted = [i32([0, 0]) for _ in pair]
        for t, s in zip(pair, starts):
            restore(t.c, s)
        torch.cuda.synchronize()
        for i in range(3):
            for j, t in enumerate(pair):
                with torch.cuda.stream(streams[j] if side else torch.cuda.current_stream()):
                    decode(t, *ins[j][i], outs[j][i], add, granted[j], new_pos, budget)
        torch.cuda.synchronize()
        results.append(([snapshot(t.c) for t in pair], outs))
    for j, t in enumerate(pair):
        a, b = results[0][0][j], results[1][0][j]
        same(a, b, a["len"].tolist(), t.cap)
        assert torch.equal(a["pool"], b["pool"])
        assert all(torch.equal(x, y) for x, y in zip(results[0][1][j], results[1][1][j]))


@pytest.mark.parametrize("hq,hkv,d,page_rows,dtype,lens", [
    (4, 2, 64, 16, "f32", [51, 16, 1, 0, 48]), (7, 1, 128, 32, "bf16", [96, 33, 0, 64, 95]), (32, 2, 128, 16, "f32", [700, 3, 688, 64, 0]),
    (512, 128, 128, 16, "bf16", [200, 1, 16, 0, 207]), (32, 4, 128, 32, "f32", [3341, 0, 257, 1, 2049])])
def test_guard_bands(hq, hkv, d, page_rows, dtype, lens):
    """No call writes outside its buffers: each lies between guard bands, the last page of the pool and the last row of a slot
    in use, the workspace of the size asked for."""
    from test_gpu_guards import Guarded, check_guards

    Guarded.registry = []
    layers, batch = 2, len(lens)
    max_pages = -(-max(lens) // page_rows)
    cap, used = max_pages * page_rows, sum(-(-n // page_rows) for n in lens)
    s = B.make_q4_shape(batch, layers, hq, hkv, d, page_rows, used + 2 * max_pages, max_pages, dtype)
    def buffer(name, dims, t=torch.int32, fill=0):
        g = Guarded(name, dims, t)
        g.t.fill_(fill)
        return g.t
    pool = buffer("pool", (B.kv_q4_pool_bytes(s),), torch.uint8, 255)
    c = B.KvQ4Cache(s, pool, buffer("table", (batch, max_pages), fill=-1), buffer("len", (batch,)), buffer("refs", (s.n_pages,)),
                    buffer("u", (batch, cap), torch.float32), buffer("pos", (batch, cap)))
    ws = buffer("ws", (B.kv_q4_workspace_bytes(s, cap, layers),), torch.uint8)
    add, granted, new_pos = buffer("add", (batch,)), buffer("granted", (batch,)), buffer("new_pos", (batch,))
    add.copy_(i32(lens))
    q, o = (buffer(n, (layers, batch, hq, d), DT[dtype]) for n in ("q", "o"))
    q.copy_(torch.randn(q.shape, generator=gen(1)))
    k, v, k2, v2 = (buffer(n, (layers, batch, hkv, max(lens), d), DT[dtype]) for n in ("k", "v", "k2", "v2"))
    k.copy_(torch.randn(k.shape, generator=gen(2)))
    v.copy_(torch.randn(v.shape, generator=gen(3)))
    scores, u_out = buffer("s", (layers, batch, cap), torch.float32), buffer("u_out", (batch, cap), torch.float32)
    keep, budget = buffer("keep", (batch, cap), torch.uint8), buffer("budget", (batch,))
    def run(name, *args, **kw):
        getattr(B, name)(c, *args, ws, **kw)
        check_guards(name)
    run("kv_q4_reserve", add, new_pos, granted=granted)
    assert granted.tolist() == lens and B.faults(ws) == 0
    run("kv_q4_store", 0, layers, max(lens), k, v, count=granted)
    run("kv_q4_load", 0, layers, max(lens), k2, v2, count=granted)
    for count in (1, layers):
        run("kv_q4_attend", 0, count, cap, q, o, s_out=scores, alpha=0.5, u_prior=c.u, u_out=u_out)
    run("kv_q4_attend", 0, layers, cap, q, o)
    c.u.copy_(torch.rand(c.u.shape, generator=gen(4)))
    empty = lens.index(0)
    run("kv_q4_fork", i32([0]), i32([empty]))
    budget.copy_(i32([n - 1 if b else n // 2 for b, n in enumerate(lens)]).clamp(min=0))
    budget[empty] = max(lens[0] - 2, 1)
    run("kv_q4_evict", cap, budget, keep_out=keep)
    run("kv_q4_compact", cap, keep)
    run("kv_q4_free", i32(list(range(batch))))
    assert B.faults(ws) == 0 and not c.refs.any() and not c.len.any()


# ---- borders of the arguments -------------------------------------------------------------------------------

@pytest.mark.parametrize("hq,hkv", [(4, 1), (10, 2), (6, 1), (16, 2), (9, 1), (16, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_probabilities_keep_32_bits(hq, hkv, d):
    """bf16 outputs are the exact ones rounded once, but for sums and exponentials in 32 bits.

    A query has one element, so a logit is one product, exact but for its scaling: off by 2^-23 of itself in base 2, a
    probability by ln 2 of both logits' errors and of the subtraction's (2^-24 of it), and the exponential's 2^-23.  Eight rows: as
    many additions in the products and in the sum (2^-23 each at most), and 8 roundings more.  The output's own rounding: half a
    step of the exact value."""
    batch, n = 24, 8
    t = Cache([n] * batch, hq=hq, hkv=hkv, d=d)
    levels = torch.tensor([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    k = torch.zeros(1, batch, hkv, n, d)
    k[..., 0] = levels[torch.randint(0, 7, (1, batch, hkv, n), generator=gen(1))]
    v = torch.randn(1, batch, hkv, n, d, generator=gen(2))
    B.kv_q4_store(t.c, 0, 1, n, k.bfloat16().cuda(), v.bfloat16().cuda(), t.ws)
    q = torch.zeros(1, batch, hq, d)
    q[..., 0] = 1.0 + 2.0 * torch.rand(1, batch, hq, generator=gen(3))
    q = q.bfloat16().cuda()
    o = torch.empty_like(q)
    B.kv_q4_attend(t.c, 0, 1, n, q, o, t.ws)
    for b in range(batch):
        want, _, size, av = R.attend(q[0, b].double().cpu().numpy(), *t.values(0, b))
        z = size * 1.4427
        rel = 2 * (0.6932 * (2 * z * 2.0 ** -23 + z * 2.0 ** -24) + 2.0 ** -23) + (2 * n + 8) * 2.0 ** -23
        step = 2.0 ** (np.floor(np.log2(np.abs(want) + rel * av)) - 8)
        assert (np.abs(o[0, b].double().cpu().numpy() - want) <= step + rel * av).all(), b


def test_utilities_swapped_after_the_fold():
    """The utilities that a fold wrote elsewhere take the place of the old ones, whose memory goes to something else."""
    t = Cache([40, 33], hq=4, hkv=2, page_rows=16).fill()
    q = torch.randn(1, 2, 4, 128, generator=gen(3)).bfloat16().cuda()
    o, out = torch.empty_like(q), torch.zeros_like(t.c.u)
    B.kv_q4_attend(t.c, 0, 1, t.cap, q, o, t.ws, alpha=0.5, u_prior=t.c.u, u_out=out)
    t.c.u.fill_(float("nan"))
    t.c.u = out
    u, pos = out.cpu().numpy().astype(np.float64), t.c.pos.cpu().numpy()
    keep = torch.zeros(2, t.cap, dtype=torch.uint8, device="cuda")
    B.kv_q4_evict(t.c, t.cap, i32([7, 20]), t.ws, keep_out=keep)
    for b, (n, m) in enumerate(((40, 7), (33, 20))):
        want = np.zeros(n, dtype=np.uint8)
        want[np.lexsort((pos[b, :n], -u[b, :n]))[:m]] = 1
        assert np.array_equal(keep[b, :n].cpu().numpy(), want)
    assert t.faults() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_counts_beyond_the_rows(dtype):
    """A count above the call's rows, or below 0, is reported; the rows that the call does have are stored and loaded."""
    t = Cache([40, 20, 33, 7], dtype=dtype)
    k, v = (torch.randn(1, 4, 2, 4, 128, generator=gen(i)).to(DT[dtype]).cuda() for i in (1, 2))
    before = t.c.pool.clone()
    for bad, left in ((i32([6, 0, 4, 3]), 34), (i32([4, -1, 4, 3]), 36)):
        t.c.pool.copy_(before)
        B.kv_q4_store(t.c, 0, 1, 4, k, v, t.ws, count=bad)
        assert t.faults() == B.KV_FAULT_CACHE
        got, _ = t.values(0, 0)  # rows len - count ...: the first four of them
        assert np.array_equal(got[:, left : left + 4], R.fast_values(k[0, 0].double().cpu().numpy()))
        own = t.c.table[1, :2].long()
        assert torch.equal(t.c.pool.view(t.shape.n_pages, -1)[own], before.view(t.shape.n_pages, -1)[own])
        y = torch.full_like(k, 7.0)
        B.kv_q4_load(t.c, 0, 1, 4, y, y.clone(), t.ws, count=bad)
        assert t.faults() == B.KV_FAULT_CACHE
        assert np.array_equal(y[0, 0].double().cpu().numpy(), got[:, left : left + 4]) and (y[0, 1] == 7.0).all() and (y[0, 3, :, 3] == 7.0).all()
    B.kv_q4_store(t.c, 0, 1, 4, k, v, t.ws, count=i32([4, 0, 1, 3]))
    assert t.faults() == 0


def test_fork_refused_by_state_beside_others():
    """Destinations in use and a source whose table names no page, among forks that are good: each workgroup of the call goes its own
    way after the second check, whichever of its waves get there first."""
    t = Cache([1000, 700, 5, 0, 0, 0, 16, 0, 0], layers=1, hq=1, hkv=1, d=64, max_pages=2100, n_pages=130)
    t.c.table[1, 43] = t.shape.n_pages
    table, refs = t.c.table.clone(), t.c.refs.clone()
    for _ in range(3):
        B.kv_q4_fork(t.c, i32([0, 1, 0, 2, 0, 1]), i32([3, 4, 6, 5, 7, 8]), t.ws)
        assert t.faults() == B.KV_FAULT_CACHE
        assert t.c.len.tolist() == [1000, 700, 5, 1000, 0, 5, 16, 1000, 0]
        for dst, src in ((3, 0), (5, 2), (7, 0)):
            assert torch.equal(t.c.table[dst], table[src])
        assert torch.equal(t.c.table[[0, 1, 2, 4, 6, 8]], table[[0, 1, 2, 4, 6, 8]])
        B.kv_q4_free(t.c, i32([3, 5, 7]), t.ws)
        assert torch.equal(t.c.refs, refs) and t.faults() == 0


@pytest.mark.parametrize("bias", [3.0e38, -3.0e38, 2.0e38, float(torch.finfo(torch.float32).max), float(torch.finfo(torch.float32).min)])
@pytest.mark.parametrize("layers", [1, 32])
def test_bias_of_the_types_largest(bias, layers):
    """A finite bias of any size: the rows with it share all weight (or have none where others lack it), alike where it hides the
    logits; all rows of slot 1 have it, none of slot 2.  32 layers: the logits stay in LDS."""
    t = Cache([40, 33, 64, 0] * 4, layers=layers, hq=8, hkv=4, d=64, page_rows=16).fill()
    t.c.pos[:] = torch.arange(t.cap, dtype=torch.int32, device="cuda")
    q = torch.randn(layers, 16, 8, 64, generator=gen(3)).bfloat16().cuda()
    cur, window = i32([40, 10, 3000, 0] * 4), 20
    o, s = torch.full_like(q, 9.0), torch.full((layers, 16, t.cap), 9.0, device="cuda")
    B.kv_q4_attend(t.c, 0, layers, t.cap, q, o, t.ws, cur_pos=cur, recency_bias=bias, recency_window=window, s_out=s)
    assert t.faults() == 0
    for b in range(16):
        for l in range(0, layers, 5):
            k, v = t.values(l, b)
            n = k.shape[1]
            add = bias * (np.arange(n) >= int(cur[b]) - (window - 1))
            want, a, _, av = R.attend(q[l, b].double().cpu().numpy(), k, v, add)
            assert (np.abs(o[l, b].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * av).all(), (b, l)
            if n:
                assert np.allclose(s[l, b, :n].double().cpu().numpy(), a.mean(0), rtol=2.0 ** -11, atol=0), (b, l)


def test_recent_border_below_the_integers():
    """cur_pos - (window - 1) below every 32-bit number: all rows are recent, those of the largest positions no more than others."""
    t = Cache([40, 25], hq=4, hkv=2).fill()
    t.c.pos[:, ::3] = (1 << 31) - 1
    t.c.pos[:, 1::3] = -(1 << 31)
    q = torch.randn(1, 2, 4, 128, generator=gen(3)).bfloat16().cuda()
    o = torch.empty_like(q)
    cur = i32([-10, -(1 << 31)])
    B.kv_q4_attend(t.c, 0, 1, t.cap, q, o, t.ws, cur_pos=cur, recency_bias=1.5, recency_window=(1 << 31) - 1)
    check_attend(t, q, o, cur, 1.5, (1 << 31) - 1)


# ---- calls of many rounds and many chunks -------------------------------------------------------------------

def origin_of(keep):
    """The row that ends at each place: the kept rows behind the new end fill the holes before it, both ascending."""
    k = int(keep.sum())
    origin = np.arange(k)
    origin[np.nonzero(keep[:k] == 0)[0]] = k + np.nonzero(keep[k:])[0]
    return origin


@pytest.mark.parametrize("how", ["evict", "compact"])
@pytest.mark.parametrize("layers,lens,forks,hkv,d,page_rows,dtype", [
    (8, [4000, 2501, 1000], [0, 0, 1, 1, 2], 4, 128, 64, "bf16"),   # 16 workgroups a sequence and layer: a dozen rounds of 16 rows each
    (8, [3999, 2048], [0, 1, 0, 1, 0, 1], 16, 64, 32, "f32"),       # more copies a round than the workgroup has in flight
    (64, [700, 333, 129, 16], [0] * 6 + [1] * 6, 1, 64, 16, "bf16"),  # one workgroup: dozens of rounds
    (64, [515, 700], [0] * 14, 3, 128, 128, "bf16")])
def test_moves_of_many_rounds(layers, lens, forks, hkv, d, page_rows, dtype, how):
    """The keys and values of sequences whose moved rows and replaced pages take many rounds of copies, whole and partial ones."""
    src = list(range(len(lens), len(lens) + len(forks)))
    t = Cache(lens + [0] * len(forks), layers=layers, hq=hkv, hkv=hkv, d=d, page_rows=page_rows, dtype=dtype,
              spare=sum(-(-m // page_rows) for m in lens + [lens[f] for f in forks])).fill()
    B.kv_q4_fork(t.c, i32(forks), i32(src), t.ws)
    n = t.c.len.tolist()
    assert n == lens + [lens[f] for f in forks]
    rows = max(n)
    t.c.u.copy_(torch.rand(t.c.u.shape, generator=gen(4)))  # each sample ranks its rows for itself
    u, pos = t.c.u.cpu().numpy(), t.c.pos.cpu().numpy()
    old, new = ([torch.zeros(layers, len(n), hkv, rows, d, dtype=DT[dtype], device="cuda") for _ in range(2)] for _ in range(2))
    B.kv_q4_load(t.c, 0, layers, rows, *old, t.ws, first=i32([0] * len(n)), count=t.c.len)
    budget = [max(1, int(m * (0.55 - 0.04 * (b % 9)))) | 1 for b, m in enumerate(n)]
    keep = np.zeros((len(n), t.cap), dtype=np.uint8)
    for b, m in enumerate(n):
        keep[b, np.lexsort((pos[b, :m], -u[b, :m].astype(np.float64)))[: budget[b]]] = 1
    if how == "evict":
        B.kv_q4_evict(t.c, rows, i32(budget), t.ws)
    else:
        B.kv_q4_compact(t.c, rows, torch.from_numpy(keep).cuda(), t.ws)
    assert t.c.len.tolist() == budget and t.faults() == 0
    B.kv_q4_load(t.c, 0, layers, max(budget), *(x[:, :, :, : max(budget)] for x in new), t.ws, first=i32([0] * len(n)), count=t.c.len)
    for b, m in enumerate(n):
        origin = origin_of(keep[b, :m])
        at = torch.from_numpy(origin).cuda()
        for x, y in zip(old, new):
            assert torch.equal(y[:, b, :, : len(origin)], x[:, b].index_select(2, at)), b
        assert np.array_equal(t.c.u[b, : len(origin)].cpu().numpy(), u[b, origin])
        assert np.array_equal(t.c.pos[b, : len(origin)].cpu().numpy(), pos[b, origin])
    refs = torch.bincount(t.c.table[t.c.table >= 0].flatten().long(), minlength=t.shape.n_pages).to(torch.int32)
    assert torch.equal(refs, t.c.refs)


@pytest.mark.parametrize("n", [20000, 131072])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
def test_attention_in_many_chunks(n, d, dtype):
    """One slab of so many rows is cut into 79 and 512 chunks of 256 rows.  Values are the same over 128 rows and keys lean
    towards the queries in some of them, so that each chunk has its own output and maximum, and a chunk left out, or counted
    twice, shows.  Sums: 32 rows in a product, 8 waves, at most 512 chunks, each addition off by 2^-24."""
    t = Cache([n], hq=2, hkv=1, d=d, page_rows=256, dtype=dtype)
    q = torch.randn(1, 1, 2, d, generator=gen(3)).to(DT[dtype])
    span = torch.arange(n) // 128
    v = torch.randn(int(span.max()) + 1, d, generator=gen(2))[span]
    lean = torch.rand(int(span.max()) + 1, generator=gen(4))[span]
    k = 0.3 * torch.randn(n, d, generator=gen(1)) + 0.15 * lean[:, None] * q[0, 0].float().mean(0)
    B.kv_q4_store(t.c, 0, 1, n, *(x[None, None, None].to(DT[dtype]).cuda() for x in (k, v)), t.ws)
    kk, vv = t.values(0, 0)
    want, a, size, av = R.attend(q[0, 0].double().numpy(), kk, vv)
    rel = 2 * ((d + 4) * 2.0 ** -24 * size + 2.0 ** -22 * size) + (32 + 8 + 512 + 64) * 2.0 ** -24
    lim = 2.0 ** -8 * np.abs(want) + (rel + 2.0 ** -15) * av if dtype == "bf16" else (rel + 2.0 ** -23) * av
    q = q.cuda()
    for scores in (False, True):
        o, s = torch.full_like(q, 9.0), torch.full((1, 1, n), 9.0, device="cuda")
        B.kv_q4_attend(t.c, 0, 1, n, q, o, t.ws, s_out=s if scores else None)
        assert (np.abs(o[0, 0].double().cpu().numpy() - want) <= lim).all(), scores
    got = s[0, 0].double().cpu().numpy()
    assert (np.abs(got - a.mean(0)) <= (rel + 2 * 2.0 ** -24) * a.mean(0)).all() and t.faults() == 0


def test_smaller_calls_of_one_workspace():
    """Every way of dividing fewer rows and layers than the workspace was made for gives what the model gives."""
    t = Cache([1500, 3], layers=5, hq=4, hkv=2, page_rows=64).fill()
    t.ws = B.q4_workspace(t.shape, 1500, 5)
    q = torch.randn(5, 2, 4, 128, generator=gen(3)).bfloat16().cuda()
    room = torch.empty(5 * 2 * 1500, device="cuda")
    for n in (1500, 1499, 1281, 1280, 1025, 1024, 513, 512, 300, 256, 255, 1):
        t.c.len.copy_(torch.tensor([n, min(n, 3)]))
        for layers in (1, 2, 3, 4, 5):
            o, s = torch.full_like(q[:layers], 9.0), room[: layers * 2 * n].view(layers, 2, n).fill_(9.0)
            B.kv_q4_attend(t.c, 5 - layers, layers, n, q[:layers], o, t.ws, s_out=s)
            check_attend(t, q[:layers], o, s_out=s, layer0=5 - layers)


def test_thousands_of_slots():
    """More slots than a workgroup has threads: pages in the slots' order, copies on write, a call that runs out of pages, and
    attention, forks and frees of most slots at once."""
    batch = 2500
    t = Twin(batch=batch, n_pages=4300, max_pages=3, layers=1, hkv=1)
    r = np.random.RandomState(5)
    t.append([int(x) for x in r.randint(1, 20, 1100)] + [0] * (batch - 1100), [3] * batch)
    t.check()
    src, dst = list(range(1100)), list(range(1100, 2200))
    B.kv_q4_fork(t.c, i32(src), i32(dst), t.ws)
    t.m.fork(src, dst)
    t.check()
    t.append([int(x) for x in r.randint(0, 4, batch)], [40] * batch, "mean")
    t.check()
    t.set_u(1)
    budget = [int(x) for x in r.randint(0, 22, batch)]
    keep = [t.m.best(b, n) for b, n in enumerate(budget)]
    B.kv_q4_evict(t.c, t.cap, i32(budget), t.ws)
    t.m.compact(keep)
    t.check()
    granted = t.append([48 - n for n in t.m.len], [80] * batch)
    assert 0 < sum(x > 0 for x in granted) < batch
    t.check(B.KV_FAULT_NO_PAGES)
    q = torch.randn(1, batch, 1, 64, generator=gen(3)).bfloat16().cuda()
    o = torch.full_like(q, 9.0)
    B.kv_q4_attend(t.c, 0, 1, t.cap, q, o, t.ws)
    k, v = (torch.zeros(1, batch, 1, t.cap, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.kv_q4_load(t.c, 0, 1, t.cap, k, v, t.ws, first=i32([0] * batch), count=t.c.len)
    for b in range(0, batch, 7):
        n = t.m.len[b]
        want, _, _, av = R.attend(q[0, b].double().cpu().numpy(), k[0, b, :, :n].double().cpu().numpy(), v[0, b, :, :n].double().cpu().numpy())
        assert (np.abs(o[0, b].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * av).all(), b
    slots = [int(x) for x in r.permutation(batch)[:2400]]
    B.kv_q4_free(t.c, i32(slots), t.ws)
    t.m.free(slots)
    t.check()


@pytest.mark.parametrize("layers,hkv,lens", [(256, 1, [33, 70]), (256, 2, [5]), (37, 3, [100, 1, 0]), (5, 40, [77, 20]), (1, 17, [130, 64]), (17, 5, [65])])
def test_scores_of_many_layers_and_heads(layers, hkv, lens):
    """Every way of dividing layers and KV heads among the score's waves, the last turn whole or not."""
    t = Cache(lens, layers=layers, hq=2 * hkv, hkv=hkv, d=64).fill()
    q = torch.randn(layers, len(lens), 2 * hkv, 64, generator=gen(3)).bfloat16().cuda()
    o, s, out = torch.full_like(q, 9.0), torch.full((layers, len(lens), t.cap), 9.0, device="cuda"), torch.full_like(t.c.u, 5.0)
    B.kv_q4_attend(t.c, 0, layers, t.cap, q, o, t.ws, s_out=s, alpha=0.97, u_prior=t.c.u, u_out=out)
    scores = check_attend(t, q, o, s_out=s)
    for b, n in enumerate(lens):
        want = t.c.u[b, :n].double().cpu().numpy()
        for l in range(layers):
            want = 0.97 * want + 0.03 * scores[l, b, :n]
        # a layer's three roundings and its coefficients' (4 2^-24 of what is left of it: 1 / (1 - 0.97) layers count), and the scores'
        lim = 4 * 34 * 2.0 ** -24 * want + 2.0 ** -12 * want
        assert (np.abs(out[b, :n].double().cpu().numpy() - want) <= lim).all() and (out[b, n:] == 5.0).all()


@pytest.mark.parametrize("hq,d,dtype,n", [(32, 128, "bf16", 3456), (32, 128, "bf16", 3520), (32, 128, "bf16", 3904), (32, 128, "bf16", 3968),
                                          (40, 128, "bf16", 2900), (40, 128, "f32", 2600), (24, 64, "bf16", 5000)])
def test_scores_at_the_border_of_lds(hq, d, dtype, n):
    """Logits that fill a workgroup's half of the LDS with three columns a head, with two, and that do not fit: one long slot among
    short ones."""
    lens = [n] + [33] * 63
    t = Cache(lens, hq=hq, hkv=8, d=d, dtype=dtype, page_rows=64)
    for rows, first in ((n, 1), (33, 64)):
        kv = [torch.randn(1, first, 8, rows, d, generator=gen(i)).to(DT[dtype]) for i in (1, 2)]
        kv = [x.expand(1, 64, 8, rows, d) if first == 1 else x for x in kv]
        count = i32([n] + [0] * 63) if first == 1 else i32([0] + [33] * 63)
        B.kv_q4_store(t.c, 0, 1, rows, *(x.cuda() for x in kv), t.ws, count=count)
    q = torch.randn(1, 64, hq, d, generator=gen(3)).to(DT[dtype]).cuda()
    o, s = torch.full_like(q, 9.0), torch.full((1, 64, n), 9.0, device="cuda")
    B.kv_q4_attend(t.c, 0, 1, n, q, o, t.ws, s_out=s)
    check_attend(t, q, o, s_out=s)
