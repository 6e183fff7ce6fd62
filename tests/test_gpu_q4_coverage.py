"""Every row that a query sees is weighed once, however the calls of blocks of queries divide the rows.

With queries of zeros every weight is 1 / (rows seen), and with values of 0 and 1 the sums are whole numbers below 2^24, exact in any
order: an output is its row count, times the reciprocal of the number seen, rounded.  Tolerance: the reciprocal and the product 2^-24 each
of the result, the output's rounding 2^-8 (bf16) or 2^-24 (f32) of it; zeros are exact.  In the values' first 32 elements a tile of 32
rows counts for element `tile % 32`, so that a tile that is lost or weighed twice changes it by at least one in
(tiles / 32 + 1); each further element belongs to one row of the sequence (the first, the last, others anywhere), so that losing or
repeating it changes that output by its whole size."""
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
    x[:, r, r // 32 % 32] = 1.0
    for h in range(hkv):
        some = torch.randperm(n, generator=gen(100 * seed + h))
        some = torch.cat((torch.tensor([0, n - 1] if n > 1 else [0] * n, dtype=torch.int64), some[(some != 0) & (some != n - 1)]))[: d - 32]
        x[h, some, 32 + torch.arange(len(some))] = 1.0
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
    v, s = rows.double().numpy(), seen.astype(np.float64)
    want = np.repeat(np.matmul(s, v) / np.maximum(s.sum(-1), 1.0)[None, :, None], t.hq // t.hkv, axis=0)
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
