"""Rotated rows and the attention of windows and shared pages without a GPU: the interface's refusals (every call here is refused
on the host, so nothing is queued)."""
import re

import pytest
import torch

from paper_2609_03515_amd import binding as B
from test_q4_host import BIG, FAKE, INVALID, STRIDES, UNSUPPORTED, WORKSPACE, buffers, call, shape


def rotary(**kw):
    r = B.make_rotary([1.0] * 64, [i % 3 for i in range(64)])
    for name, value in kw.items():
        setattr(r, name, value)
    return r


def store(layer0=0, count=1, rows=2, first=None, counts=None, rot=None, pos=FAKE, k=FAKE, v=FAKE, ks=STRIDES, vs=STRIDES, q=FAKE, qs=STRIDES,
          out=FAKE, os=STRIDES, **kw):
    return call("kv_q4_store_rotary", layer0, count, rows, first, counts, rot or rotary(), pos, k, ks, v, vs, q, qs, out, os, **kw)


def strides(**kw):
    s = B.KvQ4Strides(1024, 512, 256, 128)
    for name, value in kw.items():
        setattr(s, name, value)
    return s


def test_rotary_refusals():
    assert store(ws=None) == WORKSPACE and store(ws_bytes=255) == WORKSPACE and store(ws=FAKE + 16) == INVALID
    assert store(layer0=-1) == INVALID and store(count=5) == INVALID and store(rows=0) == INVALID and store(rows=321) == INVALID
    assert store(k=None) == INVALID and store(v=None) == INVALID and store(pos=None) == INVALID
    assert store(q=None) == INVALID and store(out=None) == INVALID and store(qs=None) == INVALID and store(os=None) == INVALID
    assert store(q=None, out=None, qs=None, os=None, ws=None) == WORKSPACE  # (without queries)
    assert store(pos=FAKE + 2) == UNSUPPORTED and store(q=FAKE + 8) == UNSUPPORTED and store(out=FAKE + 4) == UNSUPPORTED
    assert store(k=FAKE + 8) == UNSUPPORTED and store(counts=FAKE + 2) == UNSUPPORTED and store(first=FAKE + 1) == UNSUPPORTED
    for field in ("layer", "batch", "head", "row"):
        odd = strides(**{field: 132})
        for name in ("ks", "vs", "qs", "os"):
            assert store(**{name: odd}) == UNSUPPORTED, (field, name)
        flat = strides(**{field: 0})
        assert store(os=flat, out=FAKE + 4096, count=2) == INVALID, field  # two rows into one place
        assert store(qs=flat, out=FAKE + 4096, count=2, ws=None) == WORKSPACE  # (one row read for several)
        assert store(qs=strides(**{field: 2048}), count=2) == INVALID, field  # in place, in another order
    for name, field in (("pool", None), ("len", None)):
        assert store(c=buffers(**{name: field})) == INVALID
    assert store(s=shape(head_dim=80)) == UNSUPPORTED


@pytest.mark.parametrize("kw,status", [
    (dict(dim=0), INVALID), (dict(dim=-16), INVALID), (dict(dim=144), INVALID), (dict(dim=24), UNSUPPORTED), (dict(dim=2), UNSUPPORTED),
    (dict(axes=0), INVALID), (dict(axes=5), UNSUPPORTED), (dict(axes=2), INVALID), (dict(adjacent=2), INVALID), (dict(adjacent=-1), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID)])
def test_rotary_parameters(kw, status):
    assert store(rot=rotary(**kw)) == status
    bad = rotary()
    bad.inv_freq[63] = float("inf")
    assert store(rot=bad) == INVALID
    bad.dim = 64  # (the last pairs are not used)
    assert store(rot=bad, ws=None) == WORKSPACE


def test_rotary_sizes():
    long = shape(batch=64, n_q_heads=1, n_kv_heads=1, max_pages=1 << 15)
    assert store(rows=1 << 19, s=long, ws=None) == WORKSPACE and store(rows=(1 << 19) + 1, s=long, ws=None) == UNSUPPORTED


@pytest.mark.parametrize("args", [([],), ([1.0] * 65,), ([1.0] * 8, [0] * 7), ([1.0] * 8, [-1] * 8), ([1.0] * 8, [256] * 8), ([1.0] * 8, None, "quarters")])
def test_make_rotary(args):
    with pytest.raises(B.KVError):
        B.make_rotary(*args)


def test_make_rotary_values():
    r = B.make_rotary([0.5, 0.25] * 8, [0, 2] * 8, "adjacent", 2.0)
    assert (r.dim, r.adjacent, r.axes, r.scale) == (32, 1, 3, 2.0) and list(r.inv_freq[:2]) == [0.5, 0.25] and list(r.axis[:2]) == [0, 2]
    assert B.make_rotary([1.0] * 8).axes == 1 and B.make_rotary([1.0] * 8, axes=4).axes == 4


def cpu_cache():
    s = shape()
    return B.KvQ4Cache.allocate(s, device="cpu")


def test_binding_refuses_host_memory_and_other_layouts():
    c = cpu_cache()
    k, q = torch.zeros(1, 3, 2, 4, 128, dtype=torch.bfloat16), torch.zeros(1, 3, 8, 4, 128, dtype=torch.bfloat16)
    pos, ws, rot = torch.zeros(1, 3, 4, dtype=torch.int32), torch.zeros(256, dtype=torch.uint8), B.make_rotary([1.0] * 8)
    for kw in (dict(), dict(q=q, q_out=q), dict(q=q), dict(q=k, q_out=k), dict(q=q.float(), q_out=q), dict(count=pos[0, 0, :1]),
               dict(q=q.transpose(3, 4), q_out=q)):
        with pytest.raises(B.KVError):
            B.kv_q4_store_rotary(c, 0, 1, 4, k, k, rot, pos, ws, **kw)


def window(layer0=0, layers=1, n=10, rows=2, count=None, q=FAKE, qs=STRIDES, win=4, sinks=1, o=FAKE + 4096, os=STRIDES, **kw):
    return call("kv_q4_attend_window", layer0, layers, n, rows, count, q, qs, win, sinks, o, os, **kw)


def shared(layer0=0, layers=1, n=10, group=FAKE, q=FAKE, o=FAKE + 4096, **kw):
    return call("kv_q4_attend_shared", layer0, layers, n, group, q, o, **kw)


@pytest.mark.parametrize("fn", [window, shared])
def test_attention_refusals(fn):
    assert fn(ws=None) == WORKSPACE and fn(ws_bytes=255) == WORKSPACE and fn(ws=FAKE + 16) == INVALID
    assert fn(layer0=-1) == INVALID and fn(layer0=4) == INVALID and fn(layers=0) == INVALID and fn(layer0=2, layers=3) == INVALID
    assert fn(n=0) == INVALID and fn(n=321) == INVALID and fn(q=None) == INVALID and fn(o=None) == INVALID and fn(o=FAKE) == INVALID
    assert fn(q=FAKE + 8) == UNSUPPORTED and fn(o=FAKE + 4) == UNSUPPORTED
    assert fn(s=shape(head_dim=80)) == UNSUPPORTED and fn(s=shape(n_q_heads=7)) == INVALID
    for field in ("pool", "table", "len", "refs"):
        assert fn(c=buffers(**{field: None})) == INVALID and fn(c=buffers(**{field: FAKE + 2})) == UNSUPPORTED
    assert fn(c=buffers(u=None, pos=None), ws=None) == WORKSPACE  # (neither is needed)


def test_window_refusals():
    assert window(rows=0) == INVALID and window(rows=321, ws=None) == WORKSPACE and window(rows=(1 << 27) + 1) == UNSUPPORTED and window(win=-1) == INVALID and window(sinks=-1) == INVALID
    assert window(qs=None) == INVALID and window(os=None) == INVALID and window(count=FAKE + 2) == UNSUPPORTED
    for field in ("layer", "batch", "head", "row"):
        assert window(qs=strides(**{field: 132})) == UNSUPPORTED and window(os=strides(**{field: 132})) == UNSUPPORTED
        assert window(os=strides(**{field: 0}), layers=2) == INVALID and window(qs=strides(**{field: 0}), layers=2, ws=None) == WORKSPACE
    # the largest grid that a launch can have
    big = shape(batch=1024, layers=16, n_q_heads=512, n_kv_heads=512, max_pages=1)
    assert window(layers=15, rows=1, s=big, ws=None) == WORKSPACE and window(layers=16, rows=1, s=big, ws=None) == UNSUPPORTED
    marks = shape(batch=64, layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, max_pages=1 << 14, dtype="f32")
    assert window(n=1 << 19, rows=32640, s=marks, ws=None) == WORKSPACE and window(n=1 << 19, rows=32769, s=marks, ws=None) == UNSUPPORTED


def test_shared_refusals():
    assert shared(group=None) == INVALID and shared(group=FAKE + 2) == UNSUPPORTED
    big = shape(batch=1024, layers=2, n_q_heads=1 << 16, n_kv_heads=1 << 16, max_pages=1)
    assert shared(layers=1, s=big, ws=None) == WORKSPACE and shared(layers=2, s=big, ws=None) == UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(), dict(head_dim=64, dtype="f32"), dict(n_q_heads=2), dict(n_q_heads=32), dict(page_rows=16)])
def test_workspaces(kw):
    """No call needs more than the workspace of a larger one: fewer rows, queries or layers."""
    s = shape(n_pages=5000, max_pages=4096, **kw)
    for sizes in ([(n, 3, 4) for n in (1, 100, 3278, 5000, 65536)], [(5000, r, 4) for r in (1, 2, 7, 64, 500)], [(5000, 3, n) for n in (1, 2, 3, 4)]):
        need = [B.kv_q4_window_workspace_bytes(s, *x) for x in sizes]
        assert need == sorted(need) and need[0] >= 256
    by_rows = [B.kv_q4_shared_workspace_bytes(s, n, 4) for n in (1, 100, 3278, 5000, 65536)]
    by_layers = [B.kv_q4_shared_workspace_bytes(s, 5000, n) for n in (1, 2, 3, 4)]
    assert by_rows == sorted(by_rows) and by_layers == sorted(by_layers)
    for n, rows, layers in ((1, 1, 1), (40, 1, 1), (5000, 1, 4), (65536, 2, 1), (65536, 300, 4), (3278, 7, 3)):
        for win in (0, 4, 4096):
            # one byte less than the call's own need is refused; what the sizing call gives is enough: the next check refuses
            assert window(layers=layers, n=n, rows=rows, win=win, s=s, ws=FAKE + 16, ws_bytes=B.kv_q4_window_workspace_bytes(s, 65536, 300, 4)) == INVALID
            assert window(layers=layers, n=n, rows=rows, win=win, s=s, ws=FAKE + 16, ws_bytes=B.kv_q4_window_workspace_bytes(s, n, rows, layers)) == INVALID
        assert shared(layers=layers, n=n, s=s, ws=FAKE + 16, ws_bytes=B.kv_q4_shared_workspace_bytes(s, n, layers)) == INVALID


@pytest.mark.parametrize("bad", [(0, 1, 1), (321, 1, 1), (10, 0, 1), (10, (1 << 27) + 1, 1), (10, 1, 0), (10, 1, 5)])
def test_workspace_refusals(bad):
    with pytest.raises(B.KVError):
        B.kv_q4_window_workspace_bytes(shape(), *bad)
    if bad[1] == 1:
        with pytest.raises(B.KVError):
            B.kv_q4_shared_workspace_bytes(shape(), bad[0], bad[2])


def test_binding_refuses_attention_of_other_layouts():
    c, ws = cpu_cache(), torch.zeros(1 << 20, dtype=torch.uint8)
    q = torch.zeros(1, 3, 8, 2, 128, dtype=torch.bfloat16)
    flat, group = q[:, :, :, 0].contiguous(), torch.zeros(3, dtype=torch.int32)
    for x, y, kw in ((q, q, {}), (q, q.float(), {}), (q[..., :64], q, {}), (q, q.transpose(3, 4), {}), (q, q, dict(count=group.long())), (q, q, dict(count=group[:2]))):
        with pytest.raises(B.KVError):
            B.kv_q4_attend_window(c, 0, 1, 10, 2, x, y, ws, **kw)
    for x, y, g in ((flat, flat, group), (flat.float(), flat, group), (flat, q, group), (flat, flat, group[:2]), (flat, flat, group.long()), (flat, flat, None)):
        with pytest.raises(B.KVError):
            B.kv_q4_attend_shared(c, 0, 1, 10, g, x, y, ws)


def test_registers():
    """The kernels keep the waves per SIMD that their plans count on: four with one column tile (128 of 512 registers), three with two,
    two with four, and spill next to nothing; the rotation holds nothing in memory."""
    import test_kernel_resources as K

    objs = K.code_object(open(B.LIB_PATH, "rb").read())
    seen = {k[".name"]: k for o in objs for k in K.metadata(o)["amdhsa.kernels"] if "q4_query_kernel" in k[".name"] or "q4_rotary_kernel" in k[".name"]}
    forms = {name: int(re.search(r"Li(?:64|128)ELi(\d)E", name).group(1)) for name in seen if "q4_query" in name}
    assert len(forms) == 16 and len(seen) == 20
    for name, tiles in forms.items():
        assert seen[name][".vgpr_count"] <= {1: 128, 2: 168, 4: 256}[tiles] and seen[name][".vgpr_spill_count"] <= 7, name
    assert all(k[".vgpr_spill_count"] == 0 and k[".vgpr_count"] <= 128 for name, k in seen.items() if name not in forms)


def test_window_sizes_without_marks():
    """The grid of the kernel that marks tiles bounds calls that have it: those of slots that keep positions."""
    s = shape(batch=64, layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, max_pages=1 << 14, dtype="f32")
    assert window(n=1 << 19, rows=32769, s=s, ws=None) == UNSUPPORTED
    assert window(n=1 << 19, rows=32769, s=s, c=buffers(pos=None), ws=None) == WORKSPACE
    assert window(n=1 << 19, rows=1 << 21, s=s, c=buffers(pos=None), ws=None) == UNSUPPORTED  # (2^23 blocks)
    assert window(n=1 << 19, rows=(1 << 21) - 16, s=s, c=buffers(pos=None), ws=None) == WORKSPACE
