"""Performance cases of the paged 4-bit cache's serving operators: rotated rows written into it, attention of one or many
queries in a window with sinks, and attention of samples that share pages.

The cache holds key and value rows in blocks of 32 elements: a scale byte E (the power of two 2^(E-127)) and 32 codes of
4 bits (sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6).  Its pool is
``[layers][n_pages][n_kv_heads]`` records of ``page_rows`` rows: the keys' codes, the keys' scales, the values' codes, the
values' scales.  ``table[b][j]`` names the page of sequence b's rows ``j * page_rows ...`` (in every layer), ``refs`` counts
the table entries that name a page, ``len`` the rows of each sequence.

A case's kind says what one pass does:

* ``rotary``: kv_q4_store_rotary, which rotates new keys and queries by their positions (one axis, or time, height and width)
  and stores the keys with their values, and kv_q4_load of the stored rows;
* ``window``: kv_q4_attend_window, the newest rows' queries over the rows that are not after them, inside the window or
  among the first positions (no window: over all that are not after them);
* ``shared``: kv_q4_attend_shared, one query per sequence, where the samples of a prompt share its pages but for the few
  that a sample has replaced, and each has rows of its own.

``own`` chooses between the plain forms below (elementary torch operations) and the library's calls.
"""
import math

import numpy as np
import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, kind, batch, layers, hq, hkv, d, dtype, page_rows, low, high, **more):
    """Lengths are spread over low .. high, one sequence has `high`: of the new rows (rotary), of the cached rows (window), of
    the prompts (shared)."""
    c = {"name": name, "kind": kind, "batch": batch, "layers": layers, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype,
         "page_rows": page_rows, "low": low, "high": high}
    c.update(more)
    return c


def listed():
    return [
        # one decode step's rows of every layer of an 8B-shaped decoder: a latency
        _case("rotary_decode", "rotary", 8, 32, 32, 8, 128, "bf16", 64, 1, 1, axes=1, rot=128, adjacent=False),
        # one layer of two prompts of image patches, with positions in time, height and width
        _case("rotary_patches", "rotary", 2, 1, 28, 4, 128, "bf16", 64, 5000, 8192, axes=3, rot=128, adjacent=False),
        # a ragged float32 chunk, half of each row rotated, neighbouring elements paired
        _case("rotary_f32_part", "rotary", 5, 2, 16, 8, 64, "f32", 16, 1, 777, axes=1, rot=32, adjacent=True),
        # the smallest attention: a two-layer float32 cache of at most 51 tokens
        _case("window_tiny", "window", 1, 2, 4, 2, 64, "f32", 16, 51, 51, rows=1, window=16, sinks=4, places="rows"),
        # one layer of the 8B-shaped decoder at its budget of 10% of 32k, whose kept rows lie anywhere in the context
        _case("window_8b_layer", "window", 8, 1, 32, 8, 128, "bf16", 64, 3277, 3277, rows=1, window=4096, sinks=4, places="evicted"),
        # one layer of one long sequence: few of its rows are in the window
        _case("window_long_b1", "window", 1, 1, 32, 8, 128, "bf16", 128, 131072, 131072, rows=1, window=8192, sinks=64, places="ordered"),
        # ragged chunks of prompts with 7 heads per KV head in small pages
        _case("window_chunk_ragged", "window", 5, 2, 28, 4, 128, "bf16", 16, 100, 2500, rows=333, window=512, sinks=4, places="ordered"),
        # a chunk of a prompt of 32k that attends to all before it
        _case("window_prefill", "window", 1, 1, 32, 8, 128, "bf16", 64, 32768, 32768, rows=2048, window=0, sinks=0, places="rows"),
        # small float32 pages and short sequences: launches are all there is
        _case("shared_tiny", "shared", 3, 2, 4, 2, 64, "f32", 16, 70, 70, groups=1, own=9, holes=0.0),
        # one layer of 16 samples of a prompt, as a decoder calls it
        _case("shared_layer", "shared", 16, 1, 32, 8, 128, "bf16", 64, 8192, 8192, groups=1, own=200, holes=0.0),
        # all layers of a prompt's 8 samples at a budget of 10% of 32k, with the pages that their evictions replaced
        _case("shared_evicted", "shared", 8, 32, 32, 8, 128, "bf16", 64, 3277, 3277, groups=1, own=16, holes=0.1),
        # two layers of 32 samples of three long prompts, 7 heads per KV head
        _case("shared_groups", "shared", 32, 2, 28, 4, 128, "bf16", 128, 9000, 16384, groups=3, own=64, holes=0.02),
    ]


_HEADS = ((32, 8, 128), (32, 8, 128), (28, 4, 128), (40, 8, 128), (16, 8, 64), (32, 4, 128), (4, 2, 64), (32, 2, 128), (8, 8, 64))
_MOST = {"rotary": 2 * 8192 * 36, "window": 32 * 2048 * 32768, "shared": 8 * 32 * 8 * 3277}  # of a listed case, see _cost


def _cost(c):
    """What a drawn case may not have more of than a listed one: elements moved, logits (and cached rows), cached rows."""
    wide = (2 if c["dtype"] == "f32" else 1) * c["d"] / 128.0
    if c["kind"] == "rotary":
        return c["batch"] * c["layers"] * c["high"] * (c["hq"] + 2 * c["hkv"]) * wide
    rows = c["batch"] * c["layers"] * c["hkv"] * c["high"] * wide
    if c["kind"] == "window":
        return max(c["batch"] * c["layers"] * c["hq"] * c["rows"] * c["high"] * wide, rows * 512.0)
    return rows


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("rotary", "window", "window", "shared"))
    while True:
        hq, hkv, d = rng.choice(_HEADS)
        high = log_int(1, {"rotary": 8192, "window": 131072, "shared": 16384}[kind])
        low = high if rng.random() < 0.4 else max(1, int(high * rng.random()))
        c = _case("", kind, log_int(1, 32), log_int(1, 32), hq, hkv, d, "f32" if rng.random() < 0.2 else "bf16",
                  rng.choice((16, 32, 64, 64, 128, 256)), low, high)
        del c["name"]
        if kind == "rotary":
            c["axes"] = rng.choice((1, 1, 3, 4))
            c["rot"] = rng.choice((d, d, d // 2, d // 4))
            c["adjacent"] = rng.random() < 0.3
        elif kind == "window":
            c["rows"] = 1 if rng.random() < 0.4 else log_int(2, 2048)
            c["window"] = 0 if rng.random() < 0.3 else log_int(1, 16384)
            c["sinks"] = rng.choice((0, 1, 4, 64))
            c["places"] = rng.choice(("rows", "ordered", "evicted"))
        else:
            c["groups"] = rng.randint(1, 4)
            c["own"] = log_int(1, 256)
            c["holes"] = rng.choice((0.0, 0.02, 0.1, 0.5))
        if _cost(c) <= _MOST[kind]:
            return c


# ---- the format, plainly ------------------------------------------------------------------------------------

def _quantise(x):
    """x [..., d] (f32 or f64 values) -> codes [..., d / 2] and scales [..., d / 32] as bytes.  The scaling is by powers of two
    and the comparisons are with numbers of few bits, so nothing is lost in either type."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 3 + (m >= 0.875).to(e.dtype), -100).clamp(-100, 125)  # the smallest e with top < 7 * 2^e
    y = torch.ldexp(b, -e[..., None])
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(y)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The f32 values that codes [..., d / 2] and scales [..., d / 32] stand for."""
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=codes.device)
    byte = torch.arange(256, device=codes.device)
    pair = torch.stack((level[byte & 15], level[byte >> 4]), -1)
    x = pair[codes.to(torch.int32)].flatten(-2)
    scale = torch.ldexp(torch.ones((), device=codes.device), scales.to(torch.int32) - 127)
    return (x.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _parts(case, pool):
    """Views of the pool: the keys' codes and scales, the values' codes and scales, [layers][pages][heads][rows][bytes]."""
    pr, d = case["page_rows"], case["d"]
    out, at = [], 0
    rec = pool.view(case["layers"], -1, case["hkv"], pr * 2 * (d // 2 + d // 32))
    for w in (d // 2, d // 32, d // 2, d // 32):
        out.append(rec[..., at : at + pr * w].unflatten(-1, (pr, w)))
        at += pr * w
    return out


def _record(case):
    return case["page_rows"] * 2 * (case["d"] // 2 + case["d"] // 32)


# ---- inputs -------------------------------------------------------------------------------------------------

def _lengths(low, high, seed, count):
    r = np.random.RandomState((seed * 7919 + 11) % (1 << 31))
    n = r.randint(low, high + 1, size=count)
    n[r.randint(count)] = high
    return n.astype(np.int64)


def _sizes(case, seed):
    """Rows of each sequence, its newest rows that the pass is about, and the most rows of any."""
    b = case["batch"]
    r = np.random.RandomState((seed + 5) % (1 << 31))
    if case["kind"] == "rotary":
        new = _lengths(case["low"], case["high"], seed, b)
        return r.randint(0, 200, size=b) + new, new, 200 + case["high"]
    if case["kind"] == "window":
        n = _lengths(case["low"], case["high"], seed, b)
        return n, np.minimum(n, _lengths(1, case["rows"], seed + 3, b)), case["high"]
    prompts = _lengths(case["low"], case["high"], seed, case["groups"])
    return prompts[np.arange(b) % case["groups"]] + r.randint(1, case["own"] + 1, size=b), np.ones(b, dtype=np.int64), case["high"] + case["own"]


def _tables(case, seed, n, max_pages):
    """Page numbers [batch][max_pages], -1 where there is none, and how many pages the pool has.  Shared: samples of a group
    name the same pages but for replaced ones, the one that their prompt ends in, and those of their own rows."""
    b, pr = case["batch"], case["page_rows"]
    r = np.random.RandomState((seed * 31 + 7) % (1 << 31))
    have = np.arange(max_pages)[None] < -(-n // pr)[:, None]
    alone = have.copy()
    if case["kind"] == "shared":
        prompts = _lengths(case["low"], case["high"], seed, case["groups"])
        whole = np.arange(max_pages)[None] < (prompts // pr)[:, None]  # pages that a prompt fills
        mine = whole[np.arange(b) % case["groups"]]
        alone = have & (~mine | (r.random_sample((b, max_pages)) < case["holes"]))
        common = np.where(whole, np.cumsum(whole.ravel()).reshape(whole.shape) - 1, 0)
        shared = int(whole.sum())
    else:
        common, shared = np.zeros((1, max_pages), dtype=np.int64), 0
    own_pages = shared + np.cumsum(alone.ravel()).reshape(alone.shape) - 1
    numbers = np.where(alone, own_pages, common[np.arange(b) % common.shape[0]])
    n_pages = shared + int(alone.sum()) + b + 3
    perm = r.permutation(n_pages)
    return np.where(have, perm[numbers], -1).astype(np.int32), n_pages


def _positions(case, seed, n, new, cap):
    """Positions of the cached rows (window): their numbers; or those that an eviction left, a quarter of the context with its
    first ones, a tenth of them in places where holes were filled, and the newest rows behind."""
    b = case["batch"]
    r = np.random.RandomState((seed * 17 + 3) % (1 << 31))
    pos = np.tile(np.arange(cap, dtype=np.int64), (b, 1))
    if case["places"] == "evicted":
        for i in range(b):
            old = int(n[i] - new[i])
            kept = np.arange(old) * 4 + r.randint(0, 4, size=old)
            first = min(old, case["sinks"])
            kept[:first] = np.arange(first)
            for x, y in r.randint(0, max(1, old), size=(old // 20, 2)):
                kept[x], kept[y] = kept[y], kept[x]
            pos[i, :old] = kept
            pos[i, old:] = 4 * old + np.arange(cap - old)
    return pos.astype(np.int32)


def _frequencies(case):
    """The angles' factors of the pairs, as float32 numbers, and the pairs' axes: the first pairs follow time, the others in
    equal runs the further axes (16, 24 and 24 of 64)."""
    pairs = case["rot"] // 2
    freq = (1.0 / 1e6 ** (np.arange(pairs) / pairs)).astype(np.float32)
    if case["axes"] == 1:
        return freq, np.zeros(pairs, dtype=np.int64)
    first = pairs // 4
    rest = 1 + np.arange(pairs - first) * (case["axes"] - 1) // max(1, pairs - first)
    return freq, np.concatenate((np.zeros(first, dtype=np.int64), rest))


def prepare(case, seed):
    """The pool is filled with random bytes first (what unused rows and pages hold is anything), then with quantised rows:
    keys, queries and values ~ N(0, 1), 2% of the tokens heavy hitters whose keys lean towards a direction that every query
    of the KV head shares (their logits rise by 3)."""
    b, L, hq, hkv, d, pr = (case[x] for x in ("batch", "layers", "hq", "hkv", "d", "page_rows"))
    dev, dt = "cuda", torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1_000_003 + 17)
    n, new, most = _sizes(case, seed)
    max_pages = -(-most // pr)
    table, n_pages = _tables(case, seed, n, max_pages)
    cap = max_pages * pr
    s = {"case": case, "n_pages": n_pages, "max_pages": max_pages, "cap": cap, "n_max": int(most)}
    s["table"] = torch.from_numpy(table).to(dev)
    s["len"] = torch.from_numpy(n).to(dev).to(torch.int32)
    refs = np.bincount(table[table >= 0], minlength=n_pages)
    s["refs"] = torch.from_numpy(refs).to(dev).to(torch.int32)
    s["pool"] = torch.randint(0, 256, (L * n_pages * hkv * _record(case),), generator=g, device=dev, dtype=torch.uint8)
    s["count"] = torch.from_numpy(new).to(dev).to(torch.int32)
    dirs = torch.randn(L, hkv, d, generator=g, device=dev)
    dirs = dirs / dirs.norm(dim=-1, keepdim=True) * d ** 0.25
    rows = {"rotary": case["high"], "window": case.get("rows"), "shared": 1}[case["kind"]]
    s["rows"] = int(rows)
    if case["kind"] != "rotary":
        kc, ks, vc, vs = _parts(case, s["pool"])
        used = torch.from_numpy(np.nonzero(refs)[0]).to(dev)
        for l in range(L):
            for p0 in range(0, used.numel(), 4096):
                p = used[p0 : p0 + 4096]
                heavy = torch.rand(p.numel(), 1, pr, 1, generator=g, device=dev) < 0.02
                x = torch.randn(p.numel(), hkv, pr, d, generator=g, device=dev) + 3.0 * heavy * dirs[l][None, :, None, :]
                kc[l, p], ks[l, p] = _quantise(x)
                x = torch.randn(p.numel(), hkv, pr, d, generator=g, device=dev)
                vc[l, p], vs[l, p] = _quantise(x)
    # token-major, as a projection's output is: [layers][batch][rows][heads][d] seen as [layers][batch][heads][rows][d]
    q = torch.randn(L, b, rows, hq, d, generator=g, device=dev) + dirs.repeat_interleave(hq // hkv, dim=1)[:, None, None]
    s["q"] = q.to(dt).transpose(2, 3)
    s["o"] = torch.zeros(L, b, rows, hq, d, dtype=dt, device=dev).transpose(2, 3)
    if case["kind"] == "rotary":
        s["k"] = torch.randn(L, b, rows, hkv, d, generator=g, device=dev).to(dt).transpose(2, 3)
        s["v"] = torch.randn(L, b, rows, hkv, d, generator=g, device=dev).to(dt).transpose(2, 3)
        s["k_back"] = torch.zeros(L, b, hkv, rows, d, dtype=dt, device=dev)
        s["v_back"] = torch.zeros_like(s["k_back"])
        r = torch.arange(rows, device=dev)
        base = torch.randint(0, 100_000, (b, 1), generator=g, device=dev)
        places = [r if case["axes"] == 1 else r // 576, r // 24 % 24, r % 24, r // 7]  # images of 24 x 24 patches
        s["positions"] = torch.stack([base + x[None] for x in places[: case["axes"]]]).to(torch.int32)  # [axes][batch][rows]
        freq, axis = _frequencies(case)
        s["freq"], s["axis"] = torch.from_numpy(freq.astype(np.float64)).to(dev), torch.from_numpy(axis).to(dev)
    s["pos"] = None
    if case["kind"] == "window" and case["places"] != "rows":
        s["pos"] = torch.from_numpy(_positions(case, seed, n, new, cap)).to(dev)
    if case["kind"] == "shared":
        s["group"] = torch.arange(b, dtype=torch.int32, device=dev) % case["groups"]
    if own:
        from paper_2609_03515_amd import binding as B

        shape = B.make_q4_shape(b, L, hq, hkv, d, pr, n_pages, max_pages, case["dtype"])
        s["cache"] = B.KvQ4Cache(shape, s["pool"], s["table"], s["len"], s["refs"], None, s["pos"])
        if case["kind"] == "rotary":
            freq, axis = _frequencies(case)
            s["rotary"] = B.make_rotary(freq.tolist(), axis.tolist(), pairs="adjacent" if case["adjacent"] else "halves")
            s["ws"] = B.q4_workspace(shape, s["n_max"], 1)
        elif case["kind"] == "window":
            s["ws"] = B.q4_window_workspace(shape, s["n_max"], s["rows"], L)
        else:
            s["ws"] = B.q4_shared_workspace(shape, s["n_max"], L)
    return s


# ---- the operators, plainly ---------------------------------------------------------------------------------

def _new_rows(case, s):
    """Slot, row, page and row in the page of every new row r < count."""
    r = torch.arange(s["rows"], device="cuda")
    row = (s["len"] - s["count"])[:, None].long() + r[None]
    page = s["table"].gather(1, (row // case["page_rows"]).clamp(0, s["max_pages"] - 1)).long()
    b, r = (r[None] < s["count"][:, None]).nonzero(as_tuple=True)
    return b, r, page[b, r], row[b, r] % case["page_rows"]


def _rotate(case, s, x):
    """x [layers][batch][heads][rows][d] rotated, in 64 bits: far positions' angles, and rows that are then quantised."""
    angle = s["positions"].double()[s["axis"]].permute(1, 2, 0) * s["freq"]  # [batch][rows][pairs]
    cos, sin = torch.cos(angle)[None, :, None], torch.sin(angle)[None, :, None]
    x = x.double()
    rot, rest = x[..., : case["rot"]], x[..., case["rot"] :]
    pair = rot.unflatten(-1, (-1, 2)) if case["adjacent"] else rot.unflatten(-1, (2, -1)).transpose(-1, -2)
    a, b = pair[..., 0], pair[..., 1]
    pair = torch.stack((a * cos - b * sin, a * sin + b * cos), -1)
    rot = pair.flatten(-2) if case["adjacent"] else pair.transpose(-1, -2).flatten(-2)
    return torch.cat((rot, rest), -1)


def _store_rotary(case, s):
    b, r, page, row = _new_rows(case, s)
    s["o"][:, b, :, r] = _rotate(case, s, s["q"]).to(s["o"].dtype)[:, b, :, r]
    kc, ks, vc, vs = _parts(case, s["pool"])
    for x, codes, scales in ((_rotate(case, s, s["k"]), kc, ks), (s["v"].float(), vc, vs)):
        codes[:, page, :, row], scales[:, page, :, row] = _quantise(x[:, b, :, r])
    s["k_back"][:, b, :, r] = _values(kc[:, page, :, row], ks[:, page, :, row]).to(s["k_back"].dtype)
    s["v_back"][:, b, :, r] = _values(vc[:, page, :, row], vs[:, page, :, row]).to(s["v_back"].dtype)


def _attend(case, s, seen):
    """Attention of q [layers][batch][heads][rows][d] over the rows of `seen` [batch][rows][n]; zero where there is none."""
    hq, hkv, n = case["hq"], case["hkv"], s["n_max"]
    live = torch.arange(n, device="cuda")[None] < s["len"][:, None]  # [batch][n]
    at = s["table"].clamp(min=0).long()
    kc, ks, vc, vs = _parts(case, s["pool"])

    def rows(codes, scales):  # [layers][batch][pages][heads][rows][d] -> [layers][batch][heads][n][d], zero where there is no row
        x = _values(codes[:, at], scales[:, at]).transpose(2, 3).flatten(3, 4)[..., :n, :]
        return torch.where(live[None, :, None, :, None], x, 0.0)

    q = s["q"].float().unflatten(2, (hkv, hq // hkv)).flatten(3, 4)  # [layers][batch][heads][group * rows][d]
    z = torch.matmul(q, rows(kc, ks).transpose(-1, -2)) / math.sqrt(case["d"])
    z = z.unflatten(3, (hq // hkv, -1)).masked_fill(~(seen & live[:, None])[None, :, None, None], -math.inf)
    e = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-1e30))
    del z
    a = e / e.sum(-1, keepdim=True).clamp(min=1e-30)
    del e
    return torch.matmul(a.flatten(3, 4), rows(vc, vs)).unflatten(3, (hq // hkv, -1)).flatten(2, 3)


def _attend_window(case, s):
    n, rows = s["n_max"], s["rows"]
    pos = torch.arange(n, device="cuda")[None].expand(case["batch"], n) if s["pos"] is None else s["pos"][:, :n].long()
    mine = (s["len"] - s["count"])[:, None].long() + torch.arange(rows, device="cuda")[None]  # the queries' own rows
    at = pos.gather(1, mine.clamp(max=n - 1))[:, :, None]
    seen = pos[:, None] <= at
    if case["window"]:
        seen &= (pos[:, None] > at - case["window"]) | (pos[:, None] < case["sinks"])
    there = torch.arange(rows, device="cuda")[None] < s["count"][:, None]
    o = _attend(case, s, seen)
    s["o"].copy_(torch.where(there[None, :, None, :, None], o, s["o"].float()))


def _attend_shared(case, s):
    s["o"].copy_(_attend(case, s, torch.ones(case["batch"], 1, s["n_max"], dtype=torch.bool, device="cuda")))


def run(s):
    case, L = s["case"], s["case"]["layers"]
    if own:
        from paper_2609_03515_amd import binding as B

        c, ws = s["cache"], s["ws"]
        if case["kind"] == "rotary":
            B.kv_q4_store_rotary(c, 0, L, s["rows"], s["k"], s["v"], s["rotary"], s["positions"], ws, count=s["count"], q=s["q"], q_out=s["o"])
            B.kv_q4_load(c, 0, L, s["rows"], s["k_back"], s["v_back"], ws, count=s["count"])
        elif case["kind"] == "window":
            B.kv_q4_attend_window(c, 0, L, s["n_max"], s["rows"], s["q"], s["o"], ws, window=case["window"], sinks=case["sinks"], count=s["count"])
        else:
            B.kv_q4_attend_shared(c, 0, L, s["n_max"], s["group"], s["q"][:, :, :, 0], s["o"][:, :, :, 0], ws)
    elif case["kind"] == "rotary":
        _store_rotary(case, s)
    elif case["kind"] == "window":
        _attend_window(case, s)
    else:
        _attend_shared(case, s)
    return {"q": s["o"], "k": s["k_back"], "v": s["v_back"]} if case["kind"] == "rotary" else {"o": s["o"]}


# ---- what a pass cannot do without --------------------------------------------------------------------------

def _mean(low, high, count):
    """Of _lengths."""
    return (low + high) / 2.0 + (high - (low + high) / 2.0) / count if low != high else float(high)


def work(case):
    b, L, hq, hkv, d = (case[x] for x in ("batch", "layers", "hq", "hkv", "d"))
    wide = 4 if case["dtype"] == "f32" else 2
    row = 2 * (d // 2 + d // 32)  # a key and a value row in the cache
    if case["kind"] == "rotary":  # each new row read and written dense, written and read in the cache; queries read and written
        new = _mean(case["low"], case["high"], b)
        return {"bytes": b * new * (L * (hkv * (4 * d * wide + 2 * row) + 2 * hq * d * wide) + 4.0 * case["axes"]),
                "flops": b * new * L * (hq + hkv) * 3.0 * case["rot"]}
    if case["kind"] == "window":
        n = _mean(case["low"], case["high"], b)
        new = min(n, _mean(1, case["rows"], b))
        sparse = 0.25 if case["places"] == "evicted" else 1.0  # of the positions before the newest rows, those that are cached
        sinks, window = (case["sinks"], case["window"]) if case["window"] else (0, 1 << 40)
        # rows that any query sees, and the rows that a query sees (the middle one)
        union = min(n, sinks + min(new, window + new - 1) + max(0.0, window - 1) * sparse)
        each = min(n - new / 2, sinks + min(new / 2, window) + max(0.0, window - new / 2) * sparse)
        places = 4.0 * n if case["places"] != "rows" else 0.0
        return {"bytes": b * (L * hkv * union * row + 2.0 * L * new * hq * d * wide + places), "flops": 4.0 * b * L * new * hq * d * each}
    prompt = _mean(case["low"], case["high"], case["groups"])
    groups = min(b, case["groups"])
    mine = (case["own"] + 1) / 2.0 + case["page_rows"] / 2.0 + prompt * case["holes"]  # rows that a sample has for itself
    distinct = groups * prompt * (1.0 - case["holes"] ** (b / groups)) + b * mine
    each = prompt + (case["own"] + 1) / 2.0
    return {"bytes": L * hkv * min(b * each, distinct) * row + 2.0 * L * b * hq * d * wide, "flops": 4.0 * b * L * hq * d * each}


# ---- from the definition, in 64 bits ------------------------------------------------------------------------

def _nearest64(x):
    """Blocks of 32 in 64 bits: each value's nearest representable one under the block's power of two."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.ceil(torch.log2(top / 7.0)), -100.0)
    e = torch.where((top > 0) & (top >= 7.0 * 2.0 ** e), e + 1, e)
    e = torch.where((top > 0) & (top < 7.0 * 2.0 ** (e - 1)), e - 1, e)
    scale = 2.0 ** e.clamp(-100, 125)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    y = x.abs() / scale
    up = torch.bucketize(y, level).clamp(1, 7)
    below, above = level[up - 1], level[up]
    near = torch.where((y - below < above - y) | ((y - below == above - y) & ((up - 1) % 2 == 0)), below, above)
    return (torch.copysign(near, x) * scale).flatten(-2)


def _turned64(case, s, x):
    """Each pair as a complex number times e^(i angle)."""
    pos, x = s["positions"].double(), x.double().clone()
    half = case["rot"] // 2
    freq, axis = _frequencies(case)
    for i in range(half):
        angle = pos[int(axis[i])] * float(freq[i])  # [batch][rows]
        turn = torch.polar(torch.ones_like(angle), angle)[None, :, None]
        re, im = (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + half)
        z = torch.complex(x[..., re], x[..., im]) * turn
        x[..., re], x[..., im] = z.real, z.imag
    return x


def _dense64(case, s, layer, head, rows, first_part):
    """Keys or values (f64) [rows][d] of one layer's and head's rows (page, row in page), an int64 tensor [rows][2]."""
    pr, d = case["page_rows"], case["d"]
    rec = s["pool"].view(case["layers"], -1, case["hkv"], _record(case))[layer, :, head]
    base = 0 if first_part else pr * (d // 2 + d // 32)
    e = torch.arange(d, device="cuda")
    code = rec[rows[:, :1], base + rows[:, 1:] * (d // 2) + e[None] // 2].long() >> (4 * (e % 2))[None] & 15
    scale = rec[rows[:, :1], base + pr * (d // 2) + rows[:, 1:] * (d // 32) + e[None] // 32].double() - 127
    expo, man = code >> 1 & 3, (code & 1).double()
    size = torch.where(expo == 0, 0.5 * man, (1 + 0.5 * man) * 2.0 ** (expo.double() - 1))
    return torch.where(code >= 8, -size, size) * 2.0 ** scale


def exact(case, seed):
    b, L, hq, hkv, d, pr = (case[x] for x in ("batch", "layers", "hq", "hkv", "d", "page_rows"))
    n, new, most = _sizes(case, seed)
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        live = (torch.arange(s["rows"], device="cuda")[None] < torch.from_numpy(new).cuda()[:, None])[None, :, None, :, None]
        out = {"q": _turned64(case, s, s["q"]), "k": _nearest64(_turned64(case, s, s["k"])), "v": _nearest64(s["v"].double())}
        return {name: torch.where(live, x, 0.0).cpu().numpy() for name, x in out.items()}
    if b * L * hkv > 4096:  # (a loop of some milliseconds for each)
        return None
    o = torch.zeros(L, b, hq, s["rows"], d, dtype=torch.float64, device="cuda")
    table = torch.from_numpy(_tables(case, seed, n, s["max_pages"])[0]).cuda().long()
    for i in range(b):
        m, c = int(n[i]), int(new[i])
        row = torch.arange(m, device="cuda")
        where = torch.stack((table[i, row // pr], row % pr), -1)
        hidden = torch.zeros(c, m, dtype=torch.bool, device="cuda")
        if case["kind"] == "window":
            place = row if s["pos"] is None else s["pos"][i, :m].long()
            gap = place[m - c :, None] - place[None]  # how far a row lies behind a query
            hidden = gap < 0
            if case["window"]:
                hidden |= (gap >= case["window"]) & (place[None] >= case["sinks"])
        for l in range(L):
            for h in range(hkv):
                k, v = _dense64(case, s, l, h, where, True), _dense64(case, s, l, h, where, False)
                for j in range(h * hq // hkv, (h + 1) * hq // hkv):
                    z = (s["q"][l, i, j, :c].double() @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                    o[l, i, j, :c] = torch.softmax(z, -1) @ v
    return {"o": o.cpu().numpy()}
