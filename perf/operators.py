"""Measured cases of the serving operators: pages of a cache and the attention that reads them.

Three groups, each on caches of the shapes the framework compresses (8 KV heads of
dimension 128 or 64 under 1 to 8 query heads each, contexts of a few tokens to 128k):

* ``beams``, ``verify``, ``store``: rows stored in, branched over, picked from and released
  from the pages of one pool, in round trips that leave the pool as full as they found it;
* ``tree``: attention of drafted tokens (a single token is a tree of one) over such pages;
* ``sink``: attention with a sliding window and sink tokens over contiguous keys and values,
  for a whole prompt, a chunk of one and a single token.

``run`` computes them in plain torch (float32, pages picked and filled by indexing) unless
``own`` is set, where it makes the framework's calls.  ``exact`` holds the definitions in
float64, one unit (and one page) at a time.
"""
from __future__ import annotations

import math

import torch

own = False

BF16, F32 = "bf16", "f32"


# ------------------------------------------------------------------ cases ----

def listed():
    return [
        # one layer of one prompt (8 KV heads of 2k retained tokens) branches into 4 beams,
        # each takes a token, and the beams are dropped
        dict(name="beams_layer", kind="beams", units=8, fan=4, lo=1900, hi=2100, page=64, d=128,
             dtype=BF16),
        # a whole model's cache (32 layers of 8 KV heads) under speculative decoding: 16
        # drafted tokens stored, the accepted ones kept, and those taken back again
        dict(name="verify_model", kind="verify", units=256, tokens=16, lo=1000, hi=4000, page=64,
             d=128, dtype=BF16),
        # a layer's prompt stored whole, compressed in place to the retained rows, released
        dict(name="store_layer_32k", kind="store", units=8, lo=32768, hi=32768, kept=2048,
             page=128, d=128, dtype=BF16, values=BF16),
        # compressed results of a model with adaptive budgets (float32 merged values) stored,
        # thinned to half, released; odd lengths, small pages
        dict(name="store_ragged", kind="store", units=250, lo=301, hi=3999, kept=150, page=16,
             d=64, dtype=BF16, values=F32),
        # decoding: one token over one compressed layer, where latency counts
        dict(name="decode_layer", kind="tree", units=8, group=4, tokens=1, lo=2048, hi=2048,
             page=64, d=128, dtype=BF16, window=0, n_sink=0),
        # decoding a batch of 64 sequences with adaptive budgets: ragged lengths
        dict(name="decode_batch", kind="tree", units=512, group=4, tokens=1, lo=500, hi=8000,
             page=64, d=128, dtype=BF16, window=0, n_sink=0),
        # decoding over an uncompressed 128k context, one layer
        dict(name="decode_128k", kind="tree", units=8, group=8, tokens=1, lo=131072, hi=131072,
             page=128, d=128, dtype=BF16, window=0, n_sink=0),
        # verifying trees of 32 drafted tokens over long caches of four sequences
        dict(name="tree_32k", kind="tree", units=32, group=4, tokens=32, lo=20000, hi=32768,
             page=64, d=128, dtype=BF16, window=0, n_sink=0),
        # float32 caches, small pages, odd group and tree, a sliding window over the slots
        dict(name="tree_f32", kind="tree", units=48, group=3, tokens=7, lo=5, hi=3001, page=16,
             d=64, dtype=F32, window=777, n_sink=4),
        # a 16k prompt through one layer with a 4k window and 4 sink tokens
        dict(name="prefill_16k", kind="sink", units=8, group=4, n=16384, nq=16384, d=128,
             dtype=BF16, window=4096, n_sink=4),
        # a chunk of a float32 prompt, odd sizes
        dict(name="chunk_f32", kind="sink", units=4, group=5, n=5003, nq=1001, d=64, dtype=F32,
             window=700, n_sink=9),
        # decoding a batch of 32 sequences with a 4k window over 32k tokens
        dict(name="decode_window", kind="sink", units=256, group=4, n=32768, nq=1, d=128,
             dtype=BF16, window=4096, n_sink=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["beams", "verify", "store", "tree", "tree", "sink", "sink"])
    d, dtype = rng.choice([64, 128, 128]), rng.choice([BF16, BF16, F32])
    page = rng.choice([16, 32, 64, 128, 256])
    hi = _log(rng, 8, 131072)
    lo = rng.choice([hi, max(1, int(hi * rng.random()))])
    if kind == "sink":
        n = _log(rng, 64, 16384)
        nq = rng.choice([1, n, _log(rng, 1, n)])
        most = max(1, min(64, (1 << 28) // (nq * n)))
        units, group = _log(rng, 1, most), rng.randint(1, 8)
        return dict(kind=kind, units=units, group=group, n=n, nq=nq, d=d, dtype=dtype,
                    window=rng.choice([0, _log(rng, 1, n), _log(rng, 16, 4096)]),
                    n_sink=rng.choice([0, 4, rng.randint(1, 64)]))
    if kind == "tree":
        units = _log(rng, 1, max(2, min(1024, (1 << 22) // hi)))
        tokens = rng.choice([1, rng.randint(2, 64)])
        hi = max(hi, tokens)
        return dict(kind=kind, units=units, group=rng.randint(1, 8), tokens=tokens,
                    lo=max(lo, tokens), hi=hi, page=page, d=d, dtype=dtype,
                    window=rng.choice([0, 0, _log(rng, 1, 2 * hi)]), n_sink=rng.choice([0, 4]))
    units = _log(rng, 1, max(2, min(512, (1 << 18) // hi)))
    if kind == "beams":
        return dict(kind=kind, units=units, fan=rng.randint(1, 8), lo=lo, hi=hi, page=page, d=d,
                    dtype=dtype)
    if kind == "verify":
        return dict(kind=kind, units=units, tokens=rng.randint(2, 64), lo=lo, hi=hi, page=page,
                    d=d, dtype=dtype)
    return dict(kind=kind, units=units, lo=lo, hi=hi, kept=rng.randint(1, lo), page=page, d=d,
                dtype=dtype, values=rng.choice([BF16, F32]))


# ----------------------------------------------------------------- inputs ----

def _type(name):
    return torch.bfloat16 if name == BF16 else torch.float32


def _lengths(case):
    """Ragged lengths spread evenly (by the golden ratio) over lo .. hi, the same for every seed."""
    lo, hi = case["lo"], case["hi"]
    at = torch.arange(case["units"], dtype=torch.float64) * 0.6180339887498949 + 0.5
    return lo + ((hi - lo + 1) * (at % 1.0)).floor().to(torch.int64).clamp_(max=hi - lo)


def _normal(shape, dtype, g):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for part in out.view(-1).split(1 << 28):
        part.copy_(torch.randn(part.shape, device="cuda", generator=g))
    return out


def _keys(shape, dtype, g):
    """Keys with log-normal channel scales."""
    k = _normal(shape, dtype, g)
    return k.mul_(torch.exp(0.5 * torch.randn(shape[-1], device="cuda", generator=g)).to(dtype))


def _ceil(a, b):
    return -(-a // b)


def _bits(refs):
    """The free pages (those in no table) as bits of int32 words, page p bit p % 32 of word p / 32."""
    pages = torch.zeros(_ceil(refs.numel(), 32) * 32, dtype=torch.int64, device=refs.device)
    pages[: refs.numel()] = (refs == 0).long()
    words = (pages.view(-1, 32) << torch.arange(32, device=refs.device)).sum(1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _pool(case, lens, width, slots, extra, g):
    """A pool whose first len(lens) units of `slots` hold lens rows, in pages scattered over it."""
    ps, d, dt = case["page"], case["d"], _type(case["dtype"])
    held = _ceil(lens, ps)
    used = int(held.sum())
    pages = used + extra
    order = torch.randperm(pages, device="cuda", generator=g)[:used].to(torch.int32)
    table = torch.full((slots, width), -1, dtype=torch.int32, device="cuda")
    e = torch.repeat_interleave(torch.arange(len(lens)), held)
    j = torch.arange(used) - (held.cumsum(0) - held)[e]
    table[e.cuda(), j.cuda()] = order
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order.long()] = 1
    n = torch.zeros(slots, dtype=torch.int32, device="cuda")
    n[: len(lens)] = lens.to(torch.int32).cuda()
    return {"k": _keys((pages, ps, d), dt, g), "v": _normal((pages, ps, d), dt, g),
            "table": table, "lens": n, "refs": refs, "free": _bits(refs)}


def _i32(x):
    return x.to(torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 17)
    kind, d, dt = case["kind"], case["d"], _type(case["dtype"])
    s = {"case": dict(case)}
    if kind == "sink":
        U, n = case["units"], case["n"]
        s["K"], s["V"] = _keys((U, n, d), dt, g), _normal((U, n, d), dt, g)
        s["q"] = _normal((U, case["group"], case["nq"], d), dt, g)
        return s
    # lengths in an order of the seed's
    lens = _lengths(case)[torch.randperm(case["units"], device="cuda", generator=g).cpu()]
    U, ps = case["units"], case["page"]
    if kind == "tree":
        t = case["tokens"]
        s["pool"] = _pool(case, lens, _ceil(case["hi"], ps), U, U // 8 + 1, g)
        # each drafted token continues one of those before it, or the cache itself (-1)
        heads = math.gcd(U, 8)
        pick = torch.rand((U // heads, t), device="cuda", generator=g)
        s["parents"] = (pick.sqrt() * (torch.arange(t, device="cuda") + 1)).floor().to(
            torch.int32) - 1
        s["q"] = _normal((U, case["group"], t, d), dt, g)
        return s
    if kind == "beams":
        E = U * case["fan"]
        s["pool"] = _pool(case, lens, _ceil(case["hi"] + 1, ps), U + E, 2 * E + 8, g)
        s["src"] = _i32(torch.arange(U).repeat_interleave(case["fan"]))
        s["dst"] = _i32(U + torch.arange(E))
        s["k"], s["v"] = _keys((E, 1, d), dt, g), _normal((E, 1, d), dt, g)
        return s
    if kind == "verify":
        t = case["tokens"]
        extra = 2 * U * (_ceil(t, ps) + 1)
        s["pool"] = _pool(case, lens, _ceil(case["hi"] + t, ps), U, extra, g)
        s["k"], s["v"] = _keys((U, t, d), dt, g), _normal((U, t, d), dt, g)
        s["before"] = _i32(lens)
        # accepted: a few drafted tokens in ascending order, one at least
        score = torch.rand((U, t), device="cuda", generator=g)
        s["count"] = 1 + (torch.rand(U, device="cuda", generator=g) * t).floor().to(
            torch.int32).clamp_(max=t - 1)
        order = score.argsort(1)
        order = torch.where(torch.arange(t, device="cuda") < s["count"][:, None], order, t)
        s["idx"] = (order.sort(1).values + s["before"][:, None]).to(torch.int32).contiguous()
        return s
    # store: packed rows of every unit, and the rows of each to keep
    total, kept = int(lens.sum()), case["kept"]
    held = int(_ceil(lens, ps).sum()) + U * _ceil(kept, ps)
    empty = torch.zeros(U, dtype=torch.int64)
    s["pool"] = _pool(case, empty, _ceil(case["hi"], ps), U, held + 5, g)
    s["k"], s["v"] = _keys((total, d), dt, g), _normal((total, d), _type(case["values"]), g)
    s["lens"], s["starts"] = _i32(lens), (lens.cumsum(0) - lens).cuda()
    # `kept` different rows of each unit, ascending: evenly spread with a random phase
    phase = torch.rand((U, kept), device="cuda", generator=g, dtype=torch.float64)
    step = s["lens"].double()[:, None] / kept
    at = (torch.arange(kept, device="cuda") + phase * (1 - 1e-9)) * step
    s["idx"] = at.floor().to(torch.int32)
    return s


# ------------------------------------------------------------ plain forms ----

def _flat(counts):
    """(entry, place in the entry) of counts[0] + counts[1] + ... things."""
    e = torch.repeat_interleave(torch.arange(counts.numel(), device=counts.device), counts)
    return e, torch.arange(e.numel(), device=e.device) - (counts.cumsum(0) - counts)[e]


def _take(p, unit, first, last):
    """Pages first .. last - 1 of each unit become the lowest free ones."""
    e, j = _flat((last - first).clamp(min=0))
    page = torch.argsort((p["refs"] != 0).to(torch.int32), stable=True)[: e.numel()]
    p["refs"][page] = 1
    p["table"][unit[e], first[e] + j] = page.to(torch.int32)


def _drop(p, unit, first, last):
    """Pages first .. last - 1 of each unit leave its table."""
    e, j = _flat((last - first).clamp(min=0))
    page = p["table"][unit[e], first[e] + j].long()
    p["refs"].index_add_(0, page, torch.full_like(page, -1, dtype=torch.int32))
    p["table"][unit[e], first[e] + j] = -1


def _at(p, unit, slot, ps):
    return p["table"][unit, slot // ps].long() * ps + slot % ps


def _append(p, ps, unit, k, v, counts, starts):
    before = p["lens"][unit].long()
    after = before + counts
    _take(p, unit, _ceil(before, ps), _ceil(after, ps))
    e, i = _flat(counts)
    at = _at(p, unit[e], before[e] + i, ps)
    for pages, rows in ((p["k"], k), (p["v"], v)):
        pages.view(-1, pages.shape[-1])[at] = rows[starts[e] + i].to(pages.dtype)
    p["lens"][unit] = after.to(torch.int32)


def _compact(p, ps, src, dst, keep, idx, counts, starts):
    """dst becomes rows 0 .. keep - 1 and the idx rows of src; dst None: in place."""
    before, after, full = p["lens"][src].long(), keep + counts, keep // ps
    if dst is None:
        # nothing follows a kept prefix whose last page is its own: that page stays
        tail = p["refs"][p["table"][src, full.clamp(max=p["table"].shape[1] - 1)].long()]
        stay = full + ((counts == 0) & (keep % ps != 0) & (tail == 1)).long()
    else:
        stay = full
    e, i = _flat((after - stay * ps).clamp(min=0))
    slot = stay[e] * ps + i
    pick = idx[(starts[e] + slot - keep[e]).clamp(min=0, max=idx.numel() - 1)].long()
    at = _at(p, src[e], torch.where(slot < keep[e], slot, pick), ps)
    rows = [p[x].view(-1, p[x].shape[-1])[at] for x in ("k", "v")]
    old = p["table"].clone()
    if dst is None:
        unit = src
        # the new pages are taken while the old ones are still held
        _take(p, src, stay, _ceil(after, ps))
        new = p["table"].clone()
        p["table"].copy_(old)
        _drop(p, src, stay, _ceil(before, ps))
        n, j = _flat((_ceil(after, ps) - stay).clamp(min=0))
        p["table"][src[n], stay[n] + j] = new[src[n], stay[n] + j]
    else:
        unit = dst
        n, j = _flat(stay)
        page = old[src[n], j]
        p["table"][dst[n], j] = page
        p["refs"].index_add_(0, page.long(), torch.ones_like(page))
        _take(p, dst, stay, _ceil(after, ps))
    at = _at(p, unit[e], slot, ps)
    for x, r in zip(("k", "v"), rows):
        p[x].view(-1, p[x].shape[-1])[at] = r
    p["lens"][unit] = after.to(torch.int32)


def _release(p, ps, unit):
    _drop(p, unit, torch.zeros_like(unit), _ceil(p["lens"][unit].long(), ps))
    p["lens"][unit] = 0


def _plain_pages(s):
    case, p = s["case"], s["pool"]
    ps, U = case["page"], case["units"]
    unit = torch.arange(U, device="cuda")
    if case["kind"] == "beams":
        src, dst = s["src"].long(), s["dst"].long()
        one, each = torch.ones_like(dst), torch.arange(dst.numel(), device="cuda")
        _compact(p, ps, src, dst, p["lens"][src].long(), s["src"], one * 0, one * 0)
        _append(p, ps, dst, s["k"][:, 0], s["v"][:, 0], one, each)
        _release(p, ps, dst)
    elif case["kind"] == "verify":
        t = case["tokens"]
        keep, starts = s["before"].long(), unit * t
        d = case["d"]
        _append(p, ps, unit, s["k"].view(-1, d), s["v"].view(-1, d), torch.full_like(unit, t), starts)
        _compact(p, ps, unit, None, keep, s["idx"].view(-1), s["count"].long(), starts)
        _compact(p, ps, unit, None, keep, s["idx"].view(-1), unit * 0, starts)
    else:
        kept = case["kept"]
        _append(p, ps, unit, s["k"], s["v"], s["lens"].long(), s["starts"])
        _compact(p, ps, unit, None, unit * 0, s["idx"].view(-1), torch.full_like(unit, kept),
                 unit * kept)
        _release(p, ps, unit)
    p["free"].copy_(_bits(p["refs"]))
    return dict(p)


def _attend(q, K, V, seen):
    """Softmax rows in float32: q [E, R, d] over K, V [E, L, d] where seen [E, R, L] (or fewer)."""
    w = torch.matmul(q, K.transpose(1, 2)).mul_(1.0 / math.sqrt(q.shape[-1]))
    w.masked_fill_(~seen, -math.inf)
    top = w.amax(-1, keepdim=True)
    none = top == -math.inf
    top = top.masked_fill(none, 0.0)
    total = w.sub_(top).exp_().sum(-1, keepdim=True)
    o = torch.matmul(w, V) / total.masked_fill(none, 1.0)
    return o, (top + total.log())[..., 0]


def _plain_tree(s):
    case, p, q = s["case"], s["pool"], s["q"]
    E, G, t, d = q.shape
    W, S, ps = case["window"], case["n_sink"], case["page"]
    L = p["table"].shape[1] * ps
    slot = torch.arange(L, device="cuda")
    at = _at(p, torch.arange(E, device="cuda")[:, None], slot[None], ps).clamp_(min=0)
    K, V = (p[x].view(-1, d)[at].float() for x in ("k", "v"))
    base = (p["lens"].long() - t)[:, None, None]
    # ancestors: the powers of the parent relation add up to the inverse of 1 minus it
    trees = s["parents"].long()
    step = torch.zeros((trees.shape[0], t, t + 1), device="cuda", dtype=torch.float64)
    step.scatter_(2, (trees + 1)[:, :, None], 1.0)
    eye = torch.eye(t, device="cuda", dtype=torch.float64)
    family = torch.linalg.solve_triangular(eye - step[:, :, 1:], eye.expand_as(step[:, :, 1:]),
                                           upper=False) > 0.5
    depth = family.sum(2) - 1
    family = family.repeat_interleave(E // trees.shape[0], 0)
    depth = depth.repeat_interleave(E // trees.shape[0], 0)
    pos = base + depth[:, :, None]
    node = (slot - base).expand(E, t, L)
    drafted = (node >= 0) & (node < t)
    node = node.clamp(0, t - 1)
    seen = (node == node) & (slot < base) | drafted & family.gather(2, node)
    if W:
        place = torch.where(drafted, base + depth[:, None].expand(E, t, t).gather(2, node), slot)
        seen &= (place < S) | (place > pos - W)
    V = V.masked_fill((slot >= p["lens"][:, None])[:, :, None], 0.0)
    o, lse = _attend(q.float().view(E, G * t, d), K, V, seen.repeat(1, G, 1))
    return {"o": o.view(E, G, t, d).to(q.dtype), "lse": lse.view(E, G, t)}


def _plain_sink(s):
    case, q = s["case"], s["q"]
    U, G, nq, d = q.shape
    n, W, S = case["n"], case["window"], case["n_sink"]
    j = torch.arange(n, device="cuda")
    pos = torch.arange(n - nq, n, device="cuda")[:, None]
    seen = j <= pos
    if W:
        seen &= (j < S) | (j > pos - W)
    # (one mask row per query of a head, the heads of a group below one another)
    o, lse = _attend(q.float().view(U, G * nq, d), s["K"].float(), s["V"].float(),
                     seen.repeat(G, 1))
    return {"o": o.view(U, G, nq, d).to(q.dtype), "lse": lse.view(U, G, nq)}


# -------------------------------------------------------- framework calls ----

def _own_pages(s):
    import paper_2605_31105_amd as grkv

    case, p = s["case"], s["pool"]
    pages = grkv.Pages(**p)
    if case["kind"] == "beams":
        grkv.pages_fork(pages, s["src"], s["dst"])
        grkv.pages_append(pages, s["k"], s["v"], units=s["dst"])
        grkv.pages_free(pages, s["dst"])
    elif case["kind"] == "verify":
        grkv.pages_append(pages, s["k"], s["v"])
        grkv.pages_compact(pages, s["idx"], keep=s["before"], counts=s["count"])
        grkv.pages_compact(pages, keep=s["before"])
    else:
        grkv.pages_append(pages, s["k"], s["v"], counts=s["lens"], starts=s["starts"],
                          rows=case["hi"])
        grkv.pages_compact(pages, s["idx"])
        grkv.pages_free(pages)
    return dict(p)


def _own_tree(s):
    import paper_2605_31105_amd as grkv

    case = s["case"]
    o, lse = grkv.tree_attention(s["q"], grkv.Pages(**s["pool"]), s["parents"],
                                 window=case["window"], n_sink=case["n_sink"], return_lse=True)
    return {"o": o, "lse": lse}


def _own_sink(s):
    import paper_2605_31105_amd as grkv

    case = s["case"]
    o, lse = grkv.sink_attention(s["q"], s["K"], s["V"], case["window"], case["n_sink"],
                                 return_lse=True)
    return {"o": o, "lse": lse}


def run(s):
    kind = s["case"]["kind"]
    if kind == "tree":
        return _own_tree(s) if own else _plain_tree(s)
    if kind == "sink":
        return _own_sink(s) if own else _plain_sink(s)
    return _own_pages(s) if own else _plain_pages(s)


# ------------------------------------------------------------------- work ----

def work(case):
    kind, d = case["kind"], case["d"]
    b = 2 if case["dtype"] == BF16 else 4
    row = 2 * b * d   # one key and one value
    if kind == "sink":
        U, G, n, nq, W, S = (case[k] for k in ("units", "group", "n", "nq", "window", "n_sink"))
        p = torch.arange(n - nq, n, dtype=torch.float64) + 1
        seen = p if not W else p.clamp(max=W) + (p - W).clamp(0, S)
        keys = n if not W else min(n, nq + W - 1 + S)
        return {"bytes": U * (row * keys + G * nq * (2 * b * d + 4)),
                "flops": 4.0 * d * U * G * float(seen.sum())}
    lens = _lengths(case)
    U, ps = case["units"], case["page"]
    if kind == "tree":
        G, t, W, S = (case[k] for k in ("group", "tokens", "window", "n_sink"))
        keys = lens if not W else lens.clamp(max=W + S + t)
        return {"bytes": float(row * keys.sum() + 4 * _ceil(keys, ps).sum()
                               + U * G * t * (2 * b * d + 4)),
                "flops": float(4.0 * d * G * t * (keys - t + 1).sum())}
    if kind == "beams":
        E = U * case["fan"]
        # the last, partial pages once each, the new rows, the tables
        moved = float((lens % ps).sum()) * case["fan"] + E
        return {"bytes": 2.0 * row * moved + 8.0 * case["fan"] * float(_ceil(lens, ps).sum()),
                "flops": 0.0}
    if kind == "verify":
        t = case["tokens"]
        # the drafted rows stored, those accepted (half of them) moved
        return {"bytes": 2.0 * row * U * t * 1.5 + 16.0 * U, "flops": 0.0}
    c = 4 if case["values"] == F32 else 2
    total = float(lens.sum())
    return {"bytes": total * (row + (b + c) * d) + 2.0 * row * U * case["kept"]
            + 4.0 * U * case["kept"], "flops": 0.0}


# ------------------------------------------------------------ definitions ----

class _Book:
    """Pages handed out and taken back one at a time."""

    def __init__(self, p, ps):
        self.ps = ps
        self.k, self.v = p["k"].double(), p["v"].double()
        self.table = [[x for x in r if x >= 0] for r in p["table"].tolist()]
        self.lens, self.refs = p["lens"].tolist(), p["refs"].tolist()
        self.width = p["table"].shape[1]
        self.low = 0

    def new(self):
        while self.refs[self.low]:
            self.low += 1
        self.refs[self.low] = 1
        return self.low

    def leave(self, page):
        self.refs[page] -= 1

    def where(self, u, slots):
        t = torch.tensor(self.table[u] or [0], device="cuda")
        return t[slots // self.ps], slots % self.ps

    def write(self, u, slots, k, v):
        at = self.where(u, slots)
        self.k[at], self.v[at] = k, v

    def read(self, u, slots):
        at = self.where(u, slots)
        return self.k[at], self.v[at]

    def append(self, u, k, v):
        n = self.lens[u]
        while len(self.table[u]) * self.ps < n + len(k):
            self.table[u].append(self.new())
        self.lens[u] = n + len(k)
        if len(k):
            self.write(u, torch.arange(n, n + len(k), device="cuda"), k.double(), v.double())

    def outputs(self):
        table = [r + [-1] * (self.width - len(r)) for r in self.table]
        refs = torch.tensor(self.refs, dtype=torch.int32, device="cuda")
        words = [0] * _ceil(len(self.refs), 32)
        for n, r in enumerate(self.refs):
            words[n // 32] |= (r == 0) << (n % 32)
        words = [w - (1 << 32) if w >> 31 else w for w in words]
        i32 = dict(dtype=torch.int32, device="cuda")
        return {"k": self.k, "v": self.v, "table": torch.tensor(table, **i32),
                "lens": torch.tensor(self.lens, **i32), "refs": refs,
                "free": torch.tensor(words, **i32)}


def _exact_pages(case, s):
    b = _Book(s["pool"], case["page"])
    ps = b.ps

    def rebuild(src, dst, keep, picks):
        """dst := rows 0 .. keep - 1 and the picked rows of src, as pages all taken before any is left."""
        plans = []
        for u, w, n, pick in zip(src, dst, keep, picks):
            stay = n // ps
            if u == w and not len(pick) and n % ps and b.refs[b.table[u][stay]] == 1:
                stay += 1
            pages = b.table[u][:stay]
            slots = torch.cat([torch.arange(min(stay * ps, n), n, device="cuda"), pick.long()])
            rows = b.read(u, slots) if len(slots) else None
            fresh = [b.new() for _ in range(max(0, _ceil(n + len(pick), ps) - stay))]
            plans.append((u, w, stay, pages, fresh, rows, n + len(pick)))
        for u, w, stay, pages, fresh, rows, n in plans:
            if u == w:
                for x in b.table[u][stay:]:
                    b.leave(x)
            else:
                for x in pages:
                    b.refs[x] += 1
            b.table[w], b.lens[w] = pages + fresh, n
            if rows is not None:
                b.write(w, torch.arange(stay * ps, n, device="cuda"), *rows)
        b.low = 0

    def release(units):
        for u in units:
            for x in b.table[u]:
                b.leave(x)
            b.table[u], b.lens[u] = [], 0
        b.low = 0

    none = torch.empty(0, dtype=torch.int64, device="cuda")
    U = case["units"]
    if case["kind"] == "beams":
        src, dst = s["src"].tolist(), s["dst"].tolist()
        rebuild(src, dst, [b.lens[u] for u in src], [none] * len(src))
        for i, u in enumerate(dst):
            b.append(u, s["k"][i], s["v"][i])
        release(dst)
    elif case["kind"] == "verify":
        every, keep = range(U), s["before"].tolist()
        for u in every:
            b.append(u, s["k"][u], s["v"][u])
        rebuild(every, every, keep, [s["idx"][u, :c] for u, c in enumerate(s["count"].tolist())])
        rebuild(every, every, keep, [none] * U)
    else:
        every = range(U)
        for u, n, at in zip(every, s["lens"].tolist(), s["starts"].tolist()):
            b.append(u, s["k"][at:at + n], s["v"][at:at + n])
        rebuild(every, every, [0] * U, list(s["idx"]))
        release(every)
    return b.outputs()


def _rows64(q, K, V, seen):
    w = q.double() @ K.double().t().contiguous() / math.sqrt(q.shape[1])
    w = w.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(w, 1)
    o = torch.exp(w - lse.clamp(min=-1e300)[:, None]) @ V.double()
    return o, lse


def _exact_tree(case, s):
    q, p, t, ps = s["q"], s["pool"], case["tokens"], case["page"]
    E, G, _, d = q.shape
    W, S = case["window"], case["n_sink"]
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:3], dtype=torch.float64, device="cuda")
    lens, trees = p["lens"].tolist(), s["parents"].tolist()
    for e in range(E):
        n, parents = lens[e], trees[e // (E // len(trees))]
        base = n - t
        slot = torch.arange(n, device="cuda")
        page = p["table"][e].long()[slot // ps]
        K, V = p["k"][page, slot % ps], p["v"][page, slot % ps]
        path, place = [], list(range(base))
        for i, up in enumerate(parents):
            path.append((path[up] if up >= 0 else []) + [i])
            place.append(base + len(path[i]) - 1)
        place = torch.tensor(place)
        seen = torch.zeros((t, n), dtype=torch.bool)
        for i in range(t):
            at = base + len(path[i]) - 1
            seen[i, :base] = True
            seen[i, torch.tensor(path[i]) + base] = True
            if W:
                seen[i] &= (place < S) | (place > at - W)
        seen = seen.cuda()
        for h in range(G):
            o[e, h], lse[e, h] = _rows64(q[e, h], K, V, seen)
    return {"o": o, "lse": lse}


def _exact_sink(case, s):
    q, n, nq, W, S = s["q"], case["n"], case["nq"], case["window"], case["n_sink"]
    U, G, _, d = q.shape
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:3], dtype=torch.float64, device="cuda")
    j = torch.arange(n, device="cuda")
    for a in range(0, nq, 1024):
        pos = torch.arange(n - nq + a, n - nq + min(nq, a + 1024), device="cuda")[:, None]
        last = int(pos[-1]) + 1
        seen = j[:last] <= pos
        if W:
            seen = seen & ((j[:last] < S) | (pos - j[:last] < W))
        for u in range(U):
            for h in range(G):
                o[u, h, a:a + 1024], lse[u, h, a:a + 1024] = _rows64(
                    q[u, h, a:a + 1024], s["K"][u, :last], s["V"][u, :last], seen)
    return {"o": o, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "tree":
        # (a few seconds at most: one unit at a time, thousands of them take too long)
        return _exact_tree(case, s) if case["units"] * case["tokens"] <= 16384 else None
    if case["kind"] == "sink":
        return _exact_sink(case, s)
    return _exact_pages(case, s)
