"""kv_q4_attend_shared against the definition in float64 (tolerances: test_gpu_q4_window.py, a call of several queries)."""
import numpy as np
import pytest
import torch

from test_gpu_q4 import DT, HEADS, Cache, gen, i32
from test_gpu_q4_window import limits, reference

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2609_03515_amd.binding")


def samples(prompts, fan, own, holes=0, keep=None, seed=0, **kw):
    """A cache whose slots 0 .. len(prompts) - 1 hold prompts and the others their samples in turn, through the library's own calls:
    forked, extended by up to `own` rows each, and (keep) evicted to that many rows by utilities of their own.  holes: table entries
    of each sample that are replaced by copies in pages of its own."""
    batch = len(prompts) * (fan + 1)
    pr = kw.get("page_rows", 16)
    max_pages = -(-(max(prompts) + own) // pr) + 1
    t = Cache(prompts + [0] * (batch - len(prompts)), max_pages=max_pages, n_pages=batch * max_pages + 3, **kw).fill()
    src = [i % len(prompts) for i in range(len(prompts), batch)]
    B.kv_q4_fork(t.c, i32(src), i32(list(range(len(prompts), batch))), t.ws)
    if own:
        add = torch.randint(0, own + 1, (batch,), generator=gen(seed + 1)).tolist()
        add[-1] = own
        granted = i32([0] * batch)
        B.kv_q4_reserve(t.c, i32(add), None, t.ws, granted=granted)
        kv = [torch.randn(t.layers, batch, t.hkv, own, t.d, generator=gen(seed + 2 + i)).to(DT[t.dtype]).cuda() for i in range(2)]
        B.kv_q4_store(t.c, 0, t.layers, own, *kv, t.ws, count=granted)
    if keep:
        t.c.u.copy_(torch.rand(t.c.u.shape, generator=gen(seed + 9)))
        budget = torch.where(torch.arange(batch) < len(prompts), t.c.len.cpu(), torch.tensor(keep)).to(torch.int32).cuda()
        B.kv_q4_evict(t.c, t.cap, budget, t.ws)
    if holes:
        table, refs = t.c.table.cpu(), t.c.refs.cpu()
        pool = t.c.pool.view(t.layers, t.shape.n_pages, -1)
        for b in range(len(prompts), batch):
            n = -(-int(t.c.len[b]) // pr)
            for j in torch.randperm(n, generator=gen(seed + b))[:holes].tolist():
                p = int(table[b, j])
                if refs[p] > 1:
                    new = int((refs == 0).nonzero()[0, 0])
                    pool[:, new] = torch.randint(0, 130, pool[:, new].shape, generator=gen(b * 100 + j), dtype=torch.uint8).cuda()
                    table[b, j], refs[p], refs[new] = new, refs[p] - 1, 1
        t.c.table.copy_(table)
        t.c.refs.copy_(refs)
    t.lens = t.c.len.tolist()
    t.sws = B.q4_shared_workspace(t.shape, t.cap, t.layers)
    assert t.faults() == 0
    return t


def check(t, q, o, layer0=0, faults=0, skip=()):
    lens = t.c.len.tolist()
    for l in range(q.shape[0]):
        for b, n in enumerate(lens):
            if b in skip:
                continue
            k, v = t.values(layer0 + l, b)
            want, size, av = reference(q[l, b].double().cpu().numpy()[:, None], k, v, np.ones((1, n), dtype=bool))
            got = o[l, b].double().cpu().numpy()[:, None]
            err, lim = np.abs(got - want), limits(t, want, size, av, n, 2)
            assert (err <= lim + 1e-37).all(), (l, b, n, err.max(), (err / (lim + 1e-37)).max())
    assert B.faults(t.sws, clear=True) == faults


def attend(t, group, layers=None, layer0=0, n_max=None, seed=7):
    layers = layers or t.layers
    q = torch.randn(layers, t.shape.batch, t.hq, t.d, generator=gen(seed)).to(DT[t.dtype]).cuda()
    o = torch.full_like(q, 9.0)
    B.kv_q4_attend_shared(t.c, layer0, layers, n_max or t.cap, i32(group), q, o, t.sws)
    return q, o


def own_groups(prompts, batch):
    return [b % prompts for b in range(batch)]


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
def test_every_group_of_heads(hq, hkv, d, dtype):
    t = samples([70, 33], 4, 20, holes=1, layers=2, hq=hq, hkv=hkv, d=d, dtype=dtype)
    q, o = attend(t, own_groups(2, 10))
    check(t, q, o)


@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("prompts,fan,own", [([1], 1, 0), ([16], 3, 0), ([17], 5, 1), ([300], 7, 40), ([255, 256, 257], 2, 3), ([1000, 5], 6, 100), ([2049], 2, 33)])
def test_lengths_and_pages(page_rows, prompts, fan, own):
    t = samples(prompts, fan, own, page_rows=page_rows, hq=8, hkv=2)
    q, o = attend(t, own_groups(len(prompts), t.shape.batch), n_max=max(t.lens))
    check(t, q, o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page_rows", [16, 64])
def test_evicted_samples(dtype, page_rows):
    """Samples that an eviction has left with pages of their own in any places, beside the prompt that is still whole."""
    t = samples([500, 400], 5, 30, keep=300, page_rows=page_rows, hq=8, hkv=4, dtype=dtype, layers=2)
    q, o = attend(t, own_groups(2, 12))
    check(t, q, o)


@pytest.mark.parametrize("name", ["one", "none", "any", "halves", "negative"])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (3, 1), (16, 1), (2, 2)])
def test_any_grouping_gives_the_same(name, hq, hkv):
    """The groups say what is worked on together and nothing else."""
    t = samples([90, 40, 70], 12, 25, holes=2, hq=hq, hkv=hkv, page_rows=32)
    n = t.shape.batch
    group = {"one": [5] * n, "none": list(range(n)), "any": torch.randint(0, 5, (n,), generator=gen(1)).tolist(),
             "halves": [b % 3 + 3 * (b >= n // 2) for b in range(n)], "negative": [-(b % 3) - 2 ** 31 + 2 for b in range(n)]}[name]
    q, o = attend(t, group)
    check(t, q, o)


def test_many_slots():
    """Groups of more slots than a block has, among several hundred; the slots of a group lie anywhere."""
    t = samples([40, 33, 64, 10, 90], 59, 3, hq=2, hkv=1, d=64)
    group = own_groups(5, 300)
    q, o = attend(t, group)
    check(t, q, o)
    order = torch.randperm(300, generator=gen(2)).tolist()
    q, o = attend(t, [order[b] % 7 for b in range(300)])
    check(t, q, o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_prompts(dtype):
    """Divided among workgroups: pages of all samples, and of one."""
    t = samples([5000, 3000], 3, 500, holes=5, page_rows=64, hq=4, hkv=1, dtype=dtype)
    q, o = attend(t, own_groups(2, 8))
    check(t, q, o)
    t = samples([9000], 7, 3, page_rows=128, hq=4, hkv=1, dtype=dtype)
    q, o = attend(t, [0] * 8)
    check(t, q, o)


def test_layers_and_empty_slots():
    t = samples([100, 0, 30], 3, 0, layers=4, hq=4, hkv=2)
    q, o = attend(t, own_groups(3, 12), layers=2, layer0=1)
    check(t, q, o, layer0=1)
    assert (o[:, 1::3] == 0).all()
    t.c.len.zero_()
    q, o = attend(t, own_groups(3, 12))
    assert (o == 0).all()


def test_ends_inside_one_page():
    """Slots that name the same page and use different numbers of its rows."""
    t = samples([60], 3, 0, hq=4, hkv=2, page_rows=32)
    t.c.len.copy_(i32([60, 33, 50, 32]))
    q, o = attend(t, [0] * 4)
    check(t, q, o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_numbers(dtype):
    """A sample's own NaN rows reach no other sample's outputs; the prompt's reach all."""
    t = samples([64], 5, 0, hq=8, hkv=2, page_rows=16, dtype=dtype)
    add = i32([0, 3, 3, 3, 3, 3])
    t.c.table[:, 4:] = -1
    B.kv_q4_reserve(t.c, add, None, t.ws, granted=None)
    k, v = (torch.randn(1, 6, 2, 3, 128, generator=gen(s)).to(DT[dtype]) for s in (1, 2))
    v[0, 2, 1, 1, 40] = float("nan")  # slot 2, KV head 1: elements 32 .. 63
    k[0, 4, :, 2, 0] = float("inf")   # slot 4: everything
    B.kv_q4_store(t.c, 0, 1, 3, k.cuda(), v.cuda(), t.ws, count=add)
    q, o = attend(t, [0] * 6)
    bad = torch.isnan(o[0].float()).cpu()
    want = torch.zeros_like(bad)
    want[2, 4:, 32:64] = True
    want[4] = True
    assert torch.equal(bad, want)
    check(t, q, o, skip=(2, 4))


def test_slots_and_pages_that_cannot_be():
    t = samples([64], 5, 10, hq=8, hkv=2, page_rows=16)
    table = t.c.table.clone()
    t.c.table[3, 1] = t.shape.n_pages
    t.c.len[4] = t.cap + 1
    t.c.len[5] = -1
    q, o = attend(t, [0] * 6)
    assert (o[:, 4:] == 0).all()
    t.c.len[4:] = 0
    t.c.table.copy_(table)
    check(t, q, o, faults=B.KV_FAULT_CACHE, skip=(3,))
    k, v = t.values(0, 3)
    seen = np.ones((1, k.shape[1]), dtype=bool)
    seen[:, 16:32] = False
    want, size, av = reference(q[0, 3].double().cpu().numpy()[:, None], k, v, seen)
    assert (np.abs(o[0, 3].double().cpu().numpy()[:, None] - want) <= limits(t, want, size, av, 80, 2)).all()


def test_as_the_decode_attention():
    t = samples([300, 200], 7, 50, holes=3, layers=3, hq=8, hkv=2, page_rows=32)
    q, o = attend(t, own_groups(2, 16))
    o2 = torch.zeros_like(o)
    B.kv_q4_attend(t.c, 0, 3, t.cap, q, o2, t.ws)
    assert (o.float() - o2.float()).abs().max() <= 2.0 ** -6 * o2.float().abs().max()


def test_workspace_serves_smaller_calls():
    t = samples([2000, 1500], 5, 100, holes=4, layers=5, hq=4, hkv=2, page_rows=64)
    ws = B.q4_shared_workspace(t.shape, t.cap, 5)
    guard = torch.full((ws.numel() + 4096,), 77, dtype=torch.uint8, device="cuda")
    guard[:256] = 0
    t.sws = guard[: ws.numel()]
    full = t.c.len.clone()
    for layers in (1, 2, 5):
        for n in (t.cap, 1000, 40, 1):
            t.c.len.copy_(full.clamp(max=n))
            q, o = attend(t, own_groups(2, 12), layers=layers, n_max=n)
            if layers == 2:
                check(t, q, o)
    assert (guard[ws.numel():] == 77).all()


def test_captured_and_replayed():
    """A captured call replays with other tables, lengths, groups and queries, beside a decode call on another stream."""
    t = samples([200, 150], 3, 40, layers=2, hq=8, hkv=2, page_rows=32)
    q = torch.randn(2, 8, 8, 128, generator=gen(3)).bfloat16().cuda()
    o, o2, group = torch.full_like(q, 9.0), torch.full_like(q, 9.0), i32([0] * 8)

    def call():
        B.kv_q4_attend_shared(t.c, 0, 2, t.cap, group, q, o, t.sws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    full = t.c.len.clone()
    for i, g in enumerate(([0, 1] * 4, [0] * 8, list(range(8)))):
        t.c.len.copy_((full * (3 - i) // 3).clamp(min=1))
        if i == 1:
            t.c.table.copy_(t.c.table.roll(2, 0))
            t.c.len.copy_(t.c.len.roll(2, 0))
            full = full.roll(2, 0)
        group.copy_(i32(g))
        q.copy_(torch.randn(q.shape, generator=gen(30 + i)))
        o.fill_(9.0)
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            B.kv_q4_attend(t.c, 0, 2, t.cap, q, o2, t.ws)
        check(t, q, o)
        side.synchronize()
        assert (o.float() - o2.float()).abs().max() <= 2.0 ** -6 * o2.float().abs().max()
