"""Serving on the paged 4-bit cache with its calls together: prompts in chunks, samples that share them, evictions and windows.
Each call's outputs are compared with the definition on what the cache then holds (tolerances: test_gpu_q4_rotary.py and
test_gpu_q4_window.py)."""
import pytest
import torch

import test_gpu_q4_rotary as T
import test_gpu_q4_shared as S
import test_gpu_q4_window as W
from test_gpu_q4 import DT, Cache, gen, i32, restore, same, snapshot

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2609_03515_amd.binding")


def empty_cache(batch, rows, **kw):
    t = Cache([0] * batch, **kw)
    t.wws, t.sws = B.q4_window_workspace(t.shape, t.cap, rows, t.layers), B.q4_shared_workspace(t.shape, t.cap, t.layers)
    return t


def projections(t, rows, seed):
    """Queries, keys and values of a layer's rows as one product leaves them: [layer][slot][row][heads][d], strided views of it."""
    x = torch.randn(t.layers, t.shape.batch, rows, t.hq + 2 * t.hkv, t.d, generator=gen(seed)).to(DT[t.dtype]).cuda().transpose(2, 3)
    return x[:, :, : t.hq], x[:, :, t.hq : t.hq + t.hkv], x[:, :, t.hq + t.hkv :]


def extend(t, add, new_pos, rows, rot, axes, seed):
    """The next `add` rows of every slot, layer by layer: stored rotated, and each layer's rotated queries."""
    granted = i32([0] * t.shape.batch)
    B.kv_q4_reserve(t.c, i32(add), i32(new_pos), t.ws, granted=granted, init="zero")
    assert granted.tolist() == add
    q, k, v = projections(t, rows, seed)
    places = torch.tensor(new_pos)[None, :, None] + torch.arange(rows)[None, None]
    places = torch.cat([places // (1 + 3 * i) for i in range(axes)]).to(torch.int32).cuda()  # (of several axes: time, height, ...)
    out = torch.full((t.layers, t.shape.batch, rows, t.hq, t.d), 9.0, dtype=DT[t.dtype], device="cuda").transpose(2, 3)
    for l in range(t.layers):
        B.kv_q4_store_rotary(t.c, l, 1, rows, k[l : l + 1], v[l : l + 1], rot[0], places, t.ws, count=granted, q=q[l : l + 1], q_out=out[l : l + 1])
    T.check(t, k, v, q, out, places, rot[1], rot[2], False, 1.0, add)
    return out


@pytest.mark.parametrize("hq,hkv,d,dtype,page_rows,axes,window,sinks", [
    (8, 2, 128, "bf16", 16, 1, 0, 0), (28, 4, 128, "bf16", 64, 3, 48, 4), (4, 4, 64, "bf16", 32, 1, 33, 0), (6, 2, 64, "f32", 16, 2, 0, 0), (8, 1, 128, "f32", 32, 1, 20, 7)])
def test_prompts_samples_and_evictions(hq, hkv, d, dtype, page_rows, axes, window, sinks):
    t = empty_cache(6, 40, layers=2, hq=hq, hkv=hkv, d=d, dtype=dtype, page_rows=page_rows, max_pages=-(-160 // page_rows), n_pages=6 * -(-160 // page_rows))
    rot = T.rotary(d, False, axes)
    # two prompts in chunks of unequal length
    at = [0, 0]
    for i, add in enumerate(([40, 17], [33, 40], [0, 9])):
        q = extend(t, add + [0] * 4, at + [0] * 4, 40, rot, axes, 10 * i)
        o = torch.full_like(q, 9.0)
        for l in range(t.layers):
            B.kv_q4_attend_window(t.c, l, 1, t.cap, 40, q[l : l + 1], o[l : l + 1], t.wws, window=window, sinks=sinks, count=i32(add + [0] * 4))
        W.check(t, q, o, 40, add + [0] * 4, window, sinks)
        at = [a + n for a, n in zip(at, add)]
    # two samples of each, a token at a time; the prompts' slots stay
    B.kv_q4_fork(t.c, i32([0, 1, 0, 1]), i32([2, 3, 4, 5]), t.ws)
    shared = t.c.refs.max().item()
    assert shared == 3
    group = [0, 1, 0, 1, 0, 1]
    for i in range(3):
        q = extend(t, [0, 0, 1, 1, 1, 1], at * 3, 1, rot, axes, 100 + i)[:, :, :, 0].contiguous()
        o = torch.full_like(q, 9.0)
        B.kv_q4_attend_shared(t.c, 0, t.layers, t.cap, i32(group), q, o, t.sws)
        S.check(t, q, o)
        at = [a + 1 for a in at]
    # each sample evicts rows of its own: pages part, rows lie in any order of their positions
    t.c.u.copy_(torch.rand(t.c.u.shape, generator=gen(5)))
    budget = [10 ** 6, 10 ** 6, 50, 60, 31, 1]
    B.kv_q4_evict(t.c, t.cap, i32(budget), t.ws)
    assert t.c.len.tolist() == [73, 66, 50, 60, 31, 1]
    for i in range(2):
        q = extend(t, [0, 0, 1, 1, 1, 1], at * 3, 1, rot, axes, 200 + i)
        o = torch.full_like(q, 9.0)
        counts = [0, 0, 1, 1, 1, 1]
        B.kv_q4_attend_window(t.c, 0, t.layers, t.cap, 1, q, o, t.wws, window=30, sinks=4, count=i32(counts))
        W.check(t, q, o, 1, counts, 30, 4)
        q, o = q[:, :, :, 0].contiguous(), torch.full((t.layers, 6, t.hq, t.d), 9.0, dtype=DT[t.dtype], device="cuda")
        B.kv_q4_attend_shared(t.c, 0, t.layers, t.cap, i32(group), q, o, t.sws)
        S.check(t, q, o)
        at = [a + 1 for a in at]
    assert t.faults() == 0


@pytest.mark.parametrize("page_rows", [16, 64])
def test_captured_steps(page_rows):
    """A step of all the calls in a graph, replayed between eager work with other rows added, budgets and positions: each replay leaves
    what the eager calls leave, bit for bit."""
    t = S.samples([90, 61], 3, 2, layers=2, hq=8, hkv=2, page_rows=page_rows)
    batch = t.shape.batch
    t.wws = B.q4_window_workspace(t.shape, t.cap, 1, t.layers)
    t.c.pos.copy_(torch.arange(t.cap, dtype=torch.int32).expand(batch, t.cap))
    rot = T.rotary(128, False, 1)[0]
    q, k, v = projections(t, 1, 3)
    add, granted, at, budget, group = i32([1] * batch), i32([0] * batch), i32([200] * batch), i32([50] * batch), i32(S.own_groups(2, batch))
    outs = [torch.empty(2, batch, 1, t.hq, t.d, dtype=torch.bfloat16, device="cuda").transpose(2, 3) for _ in range(3)]

    def step():
        B.kv_q4_reserve(t.c, add, at, t.ws, granted=granted, init="zero")
        B.kv_q4_store_rotary(t.c, 0, 2, 1, k, v, rot, at[None, :, None], t.ws, count=granted, q=q, q_out=outs[0])
        B.kv_q4_attend_shared(t.c, 0, 2, t.cap, group, outs[0][:, :, :, 0], outs[1][:, :, :, 0], t.sws)
        B.kv_q4_attend_window(t.c, 0, 2, t.cap, 1, outs[0], outs[2], t.wws, window=40, sinks=3)
        B.kv_q4_evict(t.c, t.cap, budget, t.ws)

    start = snapshot(t.c)
    step()
    torch.cuda.synchronize()
    restore(t.c, start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        if rep == 2:
            add.copy_(i32([i % 2 for i in range(batch)]))
            budget.copy_(i32([20 + 9 * i for i in range(batch)]))
            at.copy_(i32([100 + i for i in range(batch)]))
        results = []
        for run in (step, graph.replay):
            restore(t.c, start)
            for x in outs:
                x.fill_(9.0)
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            results.append((snapshot(t.c), [x.clone() for x in outs]))
        (want, wo), (got, go) = results
        same(got, want, want["len"].tolist(), t.cap)
        assert torch.equal(got["pool"], want["pool"])
        for x, y in zip(go, wo):
            assert torch.equal(x, y)
        _ = (t.c.u * 2).sum().item()
    assert t.faults() == 0 and B.faults(t.wws) == 0 and B.faults(t.sws) == 0


def test_two_calls_at_once():
    """Both attentions of one cache on two streams, with a workspace each, give what they give alone."""
    t = S.samples([700, 300], 3, 2, layers=4, hq=8, hkv=2, page_rows=32)
    batch = t.shape.batch
    t.wws = B.q4_window_workspace(t.shape, t.cap, 20, t.layers)
    t.c.pos.copy_(torch.arange(t.cap, dtype=torch.int32).expand(batch, t.cap))
    q = torch.randn(4, batch, 8, 20, 128, generator=gen(2)).bfloat16().cuda()
    one, group = q[:, :, :, 0].contiguous(), i32(S.own_groups(2, batch))

    def calls(streams):
        o, o2 = torch.full_like(q, 9.0), torch.full_like(one, 9.0)
        torch.cuda.synchronize()
        for _ in range(5):
            B.kv_q4_attend_window(t.c, 0, 4, t.cap, 20, q, o, t.wws, window=100, sinks=4, stream=streams[0])
            B.kv_q4_attend_shared(t.c, 0, 4, t.cap, group, one, o2, t.sws, stream=streams[1])
        torch.cuda.synchronize()
        return o, o2
    alone = calls([torch.cuda.current_stream()] * 2)
    at_once = calls([torch.cuda.Stream(), torch.cuda.Stream()])
    for x, y in zip(alone, at_once):
        assert torch.equal(x, y)
    W.check(t, q, alone[0], 20, None, 100, 4)
    S.check(t, one, alone[1])


def test_graphs_that_share_a_workspace():
    """A graph of one attention and one of the other in the same workspace, replayed in turn, with a form whose workgroups need more LDS
    than the default limit met for the first time while capturing."""
    t = S.samples([130], 12, 2, layers=32, hq=16, hkv=8, d=64, page_rows=32)  # (workgroups of eight waves)
    batch = t.shape.batch
    ws = torch.zeros(max(t.sws.numel(), B.kv_q4_window_workspace_bytes(t.shape, t.cap, 70, 32)), dtype=torch.uint8, device="cuda")
    t.c.pos.copy_(torch.arange(t.cap, dtype=torch.int32).expand(batch, t.cap))
    t.sws = t.wws = ws
    q = torch.randn(32, batch, 16, 70, 64, generator=gen(2)).bfloat16().cuda()
    one, group = q[:, :, :, 3].contiguous(), i32([0] * batch)
    o, o2 = torch.empty_like(q), torch.empty_like(one)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0]):
        B.kv_q4_attend_shared(t.c, 0, 32, t.cap, group, one, o2, ws)
    with torch.cuda.graph(graphs[1]):
        B.kv_q4_attend_window(t.c, 0, 32, t.cap, 70, q, o, ws, window=40, sinks=2)
    for _ in range(3):
        o.fill_(9.0)
        o2.fill_(9.0)
        for g in graphs:
            g.replay()
        _ = (t.c.u * 2).sum().item()
        e, e2 = torch.full_like(o, 9.0), torch.full_like(o2, 9.0)
        B.kv_q4_attend_shared(t.c, 0, 32, t.cap, group, one, e2, ws)
        B.kv_q4_attend_window(t.c, 0, 32, t.cap, 70, q, e, ws, window=40, sinks=2)
        assert torch.equal(o, e) and torch.equal(o2, e2)
    S.check(t, one[:3], o2[:3])
    W.check(t, q[:3], o[:3], 70, None, 40, 2)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes: rows stored and attended to in its last pages."""
    layers, pages = 2, 1 << 17
    shape = B.make_q4_shape(3, layers, 4, 2, 128, 64, pages, 2, "bf16")
    c, cap = B.KvQ4Cache.allocate(shape), 128
    assert c.pool.numel() > 1 << 32
    wws, sws = B.q4_window_workspace(shape, cap, 8, layers), B.q4_shared_workspace(shape, cap, layers)
    last = torch.tensor([[pages - 1, pages - 4], [pages - 2, pages - 6], [pages - 3, pages - 5]], dtype=torch.int32)
    c.table.copy_(last)
    c.refs[pages - 6:] = 1
    c.len.copy_(i32([100, 65, 128]))
    k, v = [torch.randn(layers, 3, 2, 128, 128, generator=gen(i)).bfloat16().cuda() for i in (1, 2)]
    rot, freq, axis = T.rotary(128, False, 1)
    places = torch.arange(128, dtype=torch.int32).expand(1, 3, 128).contiguous().cuda()
    B.kv_q4_store_rotary(c, 0, layers, 128, k, v, rot, places, wws, first=i32([0] * 3), count=c.len)
    raw = c.pool.view(layers, pages, -1)[:, pages - 6 :].cpu().numpy()
    # the pages as a pool of their own, for the model
    small = Cache([0] * 3, layers=layers, hq=4, hkv=2, page_rows=64, max_pages=2, n_pages=6)
    small.c.pool.copy_(torch.from_numpy(raw).flatten())
    small.c.table.copy_(last - (pages - 6))
    small.c.len.copy_(c.len)
    small.c.pos = c.pos = None
    small.wws, small.sws = wws, sws
    T.check(small, k, v, None, None, places, freq, axis, False, 1.0, [100, 65, 128], first=[0] * 3)
    q = torch.randn(layers, 3, 4, 8, 128, generator=gen(4)).bfloat16().cuda()
    o = torch.full_like(q, 9.0)
    B.kv_q4_attend_window(c, 0, layers, cap, 8, q, o, wws, window=70, sinks=2)
    W.check(small, q, o, 8, None, 70, 2)
    one = q[:, :, :, 0].contiguous()
    o = torch.full_like(one, 9.0)
    B.kv_q4_attend_shared(c, 0, layers, cap, i32([0, 0, 0]), one, o, sws)
    S.check(small, one, o)
