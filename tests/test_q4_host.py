"""Paged 4-bit cache without a GPU: the interface's refusals (every call here is refused on the host, so nothing is queued)
and the reference model's own agreement."""
import ctypes

import numpy as np
import pytest
import torch

import q4_reference as R
from paper_2609_03515_amd import binding as B

FAKE = 1 << 20  # a stand-in address, never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = B.KV_ERR_INVALID_ARG, B.KV_ERR_UNSUPPORTED, B.KV_ERR_WORKSPACE
GOOD = dict(batch=3, layers=4, n_q_heads=8, n_kv_heads=2, head_dim=128, page_rows=32, n_pages=50, max_pages=10, dtype="bf16")


def shape(**kw):
    return B.make_q4_shape(**{**GOOD, **kw})


def buffers(**kw):
    return B.KvQ4Buffers(**{**{name: FAKE for name, _ in B.KvQ4Buffers._fields_}, **kw})


STRIDES = B.KvQ4Strides(1024, 512, 256, 128)
BIG = 1 << 40


def call(name, *args, s=None, c=None, ws=FAKE, ws_bytes=BIG):
    ref = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args]
    return getattr(B.load_library(), name)(ctypes.byref(s or shape()), ctypes.byref(c or buffers()), *ref, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), UNSUPPORTED), (dict(n_q_heads=7), INVALID), (dict(n_q_heads=34), UNSUPPORTED), (dict(batch=0), INVALID),
    (dict(layers=257), UNSUPPORTED), (dict(page_rows=24), UNSUPPORTED), (dict(page_rows=8), UNSUPPORTED),
    (dict(page_rows=512), UNSUPPORTED), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(dtype=5), UNSUPPORTED),
    (dict(max_pages=1 << 23), UNSUPPORTED), (dict(batch=1 << 15, max_pages=1 << 12), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED)])
def test_shapes(kw, status):
    for query in (lambda s: B.kv_q4_pool_bytes(s), lambda s: B.kv_q4_workspace_bytes(s, 10, 1)):
        with pytest.raises(B.KVError) as e:
            query(shape(**kw))
        assert e.value.status == status


def test_sizes():
    assert B.kv_q4_pool_bytes(shape()) == 4 * 50 * 2 * 32 * 136
    assert B.kv_q4_pool_bytes(shape(head_dim=64)) == 4 * 50 * 2 * 32 * 68
    for bad in ((0, 1), (321, 1), (10, 0), (10, 5)):
        with pytest.raises(B.KVError):
            B.kv_q4_workspace_bytes(shape(), *bad)
    s = shape(n_pages=5000, max_pages=4096)
    by_rows = [B.kv_q4_workspace_bytes(s, n, 4) for n in (1, 100, 3278, 5000, 131072)]
    by_layers = [B.kv_q4_workspace_bytes(s, 5000, n) for n in (1, 2, 3, 4)]
    assert by_rows == sorted(by_rows) and by_layers == sorted(by_layers)


@pytest.mark.parametrize("name,args", [
    ("kv_q4_reserve", (FAKE, FAKE, 0, FAKE)), ("kv_q4_fork", (1, FAKE, FAKE)), ("kv_q4_free", (1, FAKE)),
    ("kv_q4_compact", (10, FAKE)), ("kv_q4_evict", (10, FAKE, FAKE)),
    ("kv_q4_store", (0, 1, 2, None, None, FAKE, STRIDES, FAKE, STRIDES)),
    ("kv_q4_load", (0, 1, 2, None, None, FAKE, STRIDES, FAKE, STRIDES)),
    ("kv_q4_attend", (0, 1, 10, FAKE, FAKE, 0.5, 4, FAKE, FAKE, 0.9, FAKE, FAKE))])
def test_shared_refusals(name, args):
    assert call(name, *args, ws=None, ws_bytes=0) == WORKSPACE
    assert call(name, *args, ws_bytes=255) == WORKSPACE
    assert call(name, *args, ws=FAKE + 16) == INVALID
    for field in ("pool", "table", "len", "refs"):
        assert call(name, *args, c=buffers(**{field: None})) == INVALID, field
        assert call(name, *args, c=buffers(**{field: FAKE + 2})) == UNSUPPORTED, field
    assert call(name, *args, c=buffers(u=FAKE + 1)) == UNSUPPORTED
    assert call(name, *args, c=buffers(pool=FAKE + 4)) == UNSUPPORTED
    assert call(name, *args, s=shape(head_dim=80)) == UNSUPPORTED
    assert getattr(B.load_library(), name)(None, ctypes.byref(buffers()),
                                           *[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args], FAKE, BIG,
                                           None) == INVALID


@pytest.mark.parametrize("name", ["kv_q4_store", "kv_q4_load"])
def test_row_refusals(name):
    def rows(layer0=0, count=1, rows=2, first=None, counts=None, k=FAKE, v=FAKE, ks=STRIDES, vs=STRIDES):
        return call(name, layer0, count, rows, first, counts, k, ks, v, vs)
    assert rows(layer0=-1) == INVALID and rows(layer0=4) == INVALID and rows(layer0=3, count=2) == INVALID
    assert rows(count=0) == INVALID and rows(rows=0) == INVALID and rows(rows=321) == INVALID
    assert rows(k=None) == INVALID and rows(v=None) == INVALID
    assert rows(k=FAKE + 8) == UNSUPPORTED and rows(first=FAKE + 2) == UNSUPPORTED and rows(counts=FAKE + 2) == UNSUPPORTED
    for field in ("layer", "batch", "head", "row"):
        odd = B.KvQ4Strides(1024, 512, 256, 128)
        setattr(odd, field, 132)
        assert rows(ks=odd) == UNSUPPORTED and rows(vs=odd) == UNSUPPORTED
    if name == "kv_q4_load":  # two rows into one place
        for field, kw in (("layer", dict(count=2)), ("batch", {}), ("head", {}), ("row", {})):
            flat = B.KvQ4Strides(1024, 512, 256, 128)
            setattr(flat, field, 0)
            assert rows(vs=flat, **kw) == INVALID, field


def test_attend_refusals():
    def attend(layer0=0, count=1, n=10, q=FAKE, cur=FAKE, bias=0.5, window=4, o=FAKE, s=None, alpha=0.9, prior=None, u=None, **kw):
        return call("kv_q4_attend", layer0, count, n, q, cur, bias, window, o, s, alpha, prior, u, **kw)
    assert attend(layer0=-1) == INVALID and attend(count=0) == INVALID and attend(layer0=2, count=3) == INVALID
    assert attend(n=0) == INVALID and attend(n=321) == INVALID and attend(q=None) == INVALID and attend(o=None) == INVALID
    assert attend(window=-1) == INVALID and attend(bias=float("inf")) == INVALID and attend(bias=float("nan")) == INVALID
    assert attend(cur=None) == INVALID and attend(c=buffers(pos=None)) == INVALID
    assert attend(cur=None, bias=0.0, ws=None) == WORKSPACE  # (without a bias it is not needed)
    assert attend(u=FAKE) == INVALID and attend(u=FAKE, prior=FAKE, alpha=1.0) == INVALID
    assert attend(u=FAKE, prior=FAKE, alpha=float("nan")) == INVALID
    for kw in (dict(q=FAKE + 4), dict(o=FAKE + 8), dict(s=FAKE + 2), dict(cur=FAKE + 1), dict(u=FAKE + 2, prior=FAKE)):
        assert attend(**kw) == UNSUPPORTED, kw
    need = B.kv_q4_workspace_bytes(shape(), 10, 1)
    assert attend(ws_bytes=min(need, 600) - 345) == WORKSPACE


def test_page_refusals():
    assert call("kv_q4_reserve", None, None, 0, None) == INVALID
    for init in (-1, 3):
        assert call("kv_q4_reserve", FAKE, None, init, None) == INVALID
    assert call("kv_q4_reserve", FAKE + 1, None, 0, None) == UNSUPPORTED
    assert call("kv_q4_reserve", FAKE, None, 0, FAKE + 2) == UNSUPPORTED
    for count, src, dst, status in ((0, FAKE, FAKE, INVALID), (4, FAKE, FAKE, INVALID), (1, None, FAKE, INVALID),
                                    (1, FAKE, None, INVALID), (1, FAKE + 2, FAKE, UNSUPPORTED)):
        assert call("kv_q4_fork", count, src, dst) == status
    assert call("kv_q4_free", 0, FAKE) == INVALID and call("kv_q4_free", 4, FAKE) == INVALID
    assert call("kv_q4_free", 1, None) == INVALID and call("kv_q4_free", 1, FAKE + 1) == UNSUPPORTED
    for name in ("kv_q4_compact", "kv_q4_evict"):
        more = (None,) if name == "kv_q4_evict" else ()
        assert call(name, 0, FAKE, *more) == INVALID and call(name, 321, FAKE, *more) == INVALID
        assert call(name, 10, None, *more) == INVALID
    assert call("kv_q4_evict", 10, FAKE + 2, None) == UNSUPPORTED
    assert call("kv_q4_evict", 10, FAKE, None, c=buffers(u=None)) == INVALID
    assert call("kv_q4_evict", 10, FAKE, None, c=buffers(pos=None)) == INVALID


def test_grid_limits():
    """Calls whose grids a launch cannot have are refused; the largest that it can have get as far as the workspace's check."""
    for n, status in ((65536, WORKSPACE), (65537, UNSUPPORTED)):
        assert call("kv_q4_free", 1, FAKE, s=shape(n_q_heads=n, n_kv_heads=n), ws=None) == status
    long = shape(batch=1, layers=128, n_q_heads=2, max_pages=1 << 15)
    for name in ("kv_q4_store", "kv_q4_load"):
        for rows, status in (((1 << 20) - 1, WORKSPACE), (1 << 20, UNSUPPORTED)):
            assert call(name, 0, 128, rows, None, None, FAKE, STRIDES, FAKE, STRIDES, s=long, ws=None) == status
    def attend(s, layers, n):
        return call("kv_q4_attend", 0, layers, n, FAKE, None, 0.0, 0, FAKE, None, 0.0, None, None, s=s, ws=None)
    very_long = shape(batch=1, layers=256, n_q_heads=2, max_pages=1 << 22)
    assert attend(very_long, 3, 1 << 27) == WORKSPACE and attend(very_long, 4, 1 << 27) == UNSUPPORTED
    wide = shape(batch=1 << 13, layers=64, n_q_heads=16, n_kv_heads=16, max_pages=300)
    assert attend(wide, 63, 8193) == WORKSPACE and attend(wide, 64, 8193) == UNSUPPORTED
    assert attend(wide, 64, 8192) == WORKSPACE  # (one chunk each: nothing is joined)


def host_cache(**kw):
    return B.KvQ4Cache.allocate(shape(**kw), device="cpu")


def test_binding_checks_its_tensors():
    """Types, sizes, layouts and places that the library cannot see (CPU tensors; every call is refused before the library)."""
    c = host_cache()
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    add = torch.zeros(3, dtype=torch.int32)
    kv = torch.zeros(4, 3, 2, 5, 128, dtype=torch.bfloat16)
    q = torch.zeros(4, 3, 8, 128, dtype=torch.bfloat16)
    keep = torch.zeros(3, 320, dtype=torch.uint8)
    bad = [lambda: B.kv_q4_reserve(c, add.long(), None, ws), lambda: B.kv_q4_reserve(c, add[:2], None, ws),
           lambda: B.kv_q4_reserve(c, add, add.float(), ws),
           lambda: B.kv_q4_reserve(c, torch.zeros(6, dtype=torch.int32)[::2], None, ws),
           lambda: B.kv_q4_store(c, 0, 4, 5, kv.float(), kv, ws), lambda: B.kv_q4_store(c, 0, 4, 4, kv, kv, ws),
           lambda: B.kv_q4_store(c, 0, 3, 5, kv, kv, ws), lambda: B.kv_q4_store(c, 0, 4, 5, kv, kv.transpose(3, 4), ws),
           lambda: B.kv_q4_load(c, 0, 4, 5, kv, kv[..., :64], ws), lambda: B.kv_q4_store(c, 0, 4, 5, kv, kv, ws, count=add.long()),
           lambda: B.kv_q4_attend(c, 0, 4, 10, q.float(), q, ws), lambda: B.kv_q4_attend(c, 0, 4, 10, q, q[:3], ws),
           lambda: B.kv_q4_attend(c, 0, 4, 10, q, q, ws, s_out=torch.zeros(4, 3, 9)),
           lambda: B.kv_q4_attend(c, 0, 4, 10, q, q, ws, u_prior=c.u, u_out=c.u[:, :100]),
           lambda: B.kv_q4_fork(c, add, add[:2], ws), lambda: B.kv_q4_fork(c, add.long(), add.long(), ws),
           lambda: B.kv_q4_free(c, add.long(), ws), lambda: B.kv_q4_compact(c, 10, keep[:, :300], ws),
           lambda: B.kv_q4_evict(c, 10, add, ws, keep_out=keep.int()), lambda: B.kv_q4_evict(c, 10, add, ws.int()),
           lambda: B.KvQ4Cache(c.shape, c.pool[:-1], c.table, c.len, c.refs), lambda: B.KvQ4Cache(c.shape, c.pool, c.table.long(), c.len, c.refs),
           lambda: B.KvQ4Cache(c.shape, c.pool, c.table, c.len, c.refs[:-1])]
    for i, f in enumerate(bad):
        with pytest.raises(B.KVError) as e:
            f()
        assert e.value.status == INVALID, i


def test_host_memory_is_refused():
    """A cache, or tensors, in host memory never reach a kernel."""
    c, ws = host_cache(), torch.zeros(1 << 22, dtype=torch.uint8)
    n = torch.zeros(3, dtype=torch.int32)
    kv = torch.zeros(4, 3, 2, 5, 128, dtype=torch.bfloat16)
    q = torch.zeros(4, 3, 8, 128, dtype=torch.bfloat16)
    keep = torch.zeros(3, 320, dtype=torch.uint8)
    for f in (lambda: B.kv_q4_reserve(c, n, n, ws), lambda: B.kv_q4_store(c, 0, 4, 5, kv, kv, ws),
              lambda: B.kv_q4_load(c, 0, 4, 5, kv, kv, ws), lambda: B.kv_q4_attend(c, 0, 4, 10, q, q, ws),
              lambda: B.kv_q4_fork(c, n, n, ws), lambda: B.kv_q4_free(c, n, ws), lambda: B.kv_q4_compact(c, 10, keep, ws),
              lambda: B.kv_q4_evict(c, 10, n, ws)):
        with pytest.raises(B.KVError) as e:
            f()
        assert e.value.status == INVALID


def test_reference_quantiser():
    """The reference's two forms agree, and its error is within half the distance of the neighbouring levels."""
    r = np.random.RandomState(3)
    x = r.standard_normal((50, 64)) * 2.0 ** r.randint(-90, 90, size=(50, 1))
    x[0, :32] = 0.0
    x[1, 3], x[2, 5] = 7.0 * 2.0 ** 4, -1.75
    y = R.values(*R.quantise(x))
    assert np.array_equal(y, R.fast_values(x))
    top = np.abs(x.reshape(50, 2, 32)).max(-1)
    err = np.abs(x - y).reshape(50, 2, 32).max(-1)
    assert (err <= top / 3.5).all() and (err[top == 0] == 0).all()  # 2^e <= max |x| / 3.5
    codes, _ = R.quantise(np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, 6.0, -0.0] + [0.0] * 22]))
    assert codes[0, :10].tolist() == [0, 2, 2, 4, 4, 6, 6, 8, 7, 8]


def test_attention_registers():
    """Every instance of the 4-bit attention fits four waves per SIMD (128 of 512 registers) without spills to speak of: the
    loads in flight of fewer waves do not cover the memory's latency."""
    import test_kernel_resources as K

    objs = K.code_object(open(B.LIB_PATH, "rb").read())
    seen = {k[".name"]: k for o in objs for k in K.metadata(o)["amdhsa.kernels"] if "q4_attend_kernel" in k[".name"]}
    assert len(seen) == 16
    assert max(k[".vgpr_count"] for k in seen.values()) <= 128
    assert max(k[".vgpr_spill_count"] for k in seen.values()) <= 2


def test_a_cache_follows_its_buffers():
    """Assigning a buffer of a cache (the utilities that an attention wrote, say) is what the calls see; what does not fit is
    refused and changes nothing; the shape is the cache's own."""
    s = shape()
    c = B.KvQ4Cache.allocate(s, device="cpu")
    addresses = {name: getattr(c, name).data_ptr() for name in ("pool", "table", "len", "refs", "u", "pos")}
    assert {name: getattr(c.buffers, name) for name in addresses} == addresses
    for name, old in addresses.items():
        new = torch.zeros_like(getattr(c, name))
        setattr(c, name, new)
        assert getattr(c, name) is new and getattr(c.buffers, name) == new.data_ptr() != old
        for wrong in (new.double(), new.flatten()[:-1], torch.zeros(2 * new.numel(), dtype=new.dtype)[::2], new.to("meta")):
            with pytest.raises(B.KVError) as e:
                setattr(c, name, wrong)
            assert e.value.status == INVALID and getattr(c, name) is new and getattr(c.buffers, name) == new.data_ptr()
    for name in ("pool", "table", "len", "refs"):
        with pytest.raises(B.KVError):
            setattr(c, name, None)
    for name in ("u", "pos"):
        setattr(c, name, None)
        assert getattr(c, name) is None and getattr(c.buffers, name) is None
    s.n_pages = c.shape.max_pages = 1 << 20
    assert c.shape.n_pages == GOOD["n_pages"] and c.shape.max_pages == GOOD["max_pages"]
    with pytest.raises(AttributeError):
        c.shape = s


def test_attend_checks_the_order_of_heads():
    """Queries and outputs of the right size in another order are refused, as kv_q4_store refuses such rows (host tensors: what
    passes the check is refused for its place, with the same status, so the check is looked at by itself)."""
    c = host_cache()  # 4 layers, 3 slots, 8 query heads of 128
    good = [torch.zeros(4, 3, 8, 128), torch.zeros(2, 3, 8, 128), torch.zeros(1, 3, 8, 128), torch.zeros(3, 8, 128)]
    fits = lambda t, layers: B._q4_heads(c, t.bfloat16(), layers)
    assert fits(good[0], 4) and fits(good[0], 1) and fits(good[1], 2) and fits(good[2], 1) and fits(good[3], 1)
    assert not fits(good[1], 3) and not fits(good[3], 2)
    for shape_ in ((3, 4, 8, 128), (4, 8, 3, 128), (4, 3, 128, 8), (4 * 3, 8, 128), (4, 3, 8 * 128), (4 * 3 * 8 * 128,), (8, 3, 128), (2, 2, 3, 8, 128)):
        assert not fits(torch.zeros(*shape_), 4 if len(shape_) == 4 else 1), shape_
    assert not B._q4_heads(c, None, 1) and not B._q4_heads(c, good[0], 4) and not fits(good[0].transpose(0, 1).reshape(4, 8, 3, 128).transpose(1, 2), 4)


def test_attention_pairs_registers():
    """The attention of 6 to 8 heads a KV head keeps four waves per SIMD as well."""
    import test_kernel_resources as K

    objs = K.code_object(open(B.LIB_PATH, "rb").read())
    seen = {k[".name"]: k for o in objs for k in K.metadata(o)["amdhsa.kernels"] if "q4_attend_pairs_kernel" in k[".name"]}
    assert len(seen) == 8
    assert max(k[".vgpr_count"] for k in seen.values()) <= 128
    assert max(k[".vgpr_spill_count"] for k in seen.values()) <= 2
