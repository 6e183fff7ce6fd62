"""Rotated rows and the attention of windows and shared pages without a GPU: the interface's refusals (every call here is refused
on the host, so nothing is queued)."""
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
