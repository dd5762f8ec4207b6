"""The calls on pages against the plain model: tables, lengths, counts, free bits and
statuses equal, rows bit for bit (a stored row is its source rounded once)."""
import random

import numpy as np
import pytest

from tests.pages_model import PagesModel

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pair:
    """A pool and its model, changed together and compared after every call."""

    def __init__(self, units, max_pages, pages, ps, d, dtype, seed=0):
        import paper_2605_31105_amd as G
        self.G, self.d, self.dtype = G, d, dtype
        self.pg = G.new_pages(units, max_pages, pages, ps, d, dtype)
        # rows that no call writes keep what they held
        self.pg.k.fill_(7.0)
        self.pg.v.fill_(9.0)
        self.m = PagesModel(units, max_pages, pages, ps)
        self.gen = torch.Generator().manual_seed(seed)
        self.check([], [])

    def check(self, status, want):
        torch.cuda.synchronize()
        if torch.is_tensor(status):
            status = status.tolist()
        assert status == want, (status, want)
        table, lens, refs, free = self.m.arrays()
        assert np.array_equal(self.pg.lens.cpu().numpy(), lens)
        assert np.array_equal(self.pg.table.cpu().numpy(), table)
        assert np.array_equal(self.pg.refs.cpu().numpy(), refs)
        assert np.array_equal(self.pg.free.cpu().numpy(), free)
        k = torch.full(self.pg.k.shape, 7.0, dtype=self.dtype)
        v = torch.full(self.pg.v.shape, 9.0, dtype=self.dtype)
        for (p, r), row in self.m.data.items():
            k[p, r] = 0 if row is None else row[0]
            v[p, r] = 0 if row is None else row[1]
        assert torch.equal(self.pg.k.cpu(), k) and torch.equal(self.pg.v.cpu(), v)

    def draw(self, n, kt, vt):
        k = torch.randn((n, self.d), generator=self.gen).to(kt)
        v = torch.randn((n, self.d), generator=self.gen).to(vt)
        return k, v

    def append(self, units, counts, kt=torch.bfloat16, vt=torch.bfloat16):
        """Packed rows with counts and starts, the rows of the entries in reversed order."""
        n = sum(counts)
        k, v = self.draw(n + 3, kt, vt)
        starts, at = [0] * len(counts), 3
        for i in reversed(range(len(counts))):
            starts[i] = at
            at += counts[i]
        rows = [[(k[s + j].to(self.dtype), v[s + j].to(self.dtype)) for j in range(c)]
                for s, c in zip(starts, counts)]
        st = self.G.pages_append(self.pg, k.cuda(), v.cuda(), units=_i32(units), counts=_i32(counts),
                                 starts=torch.tensor(starts, device="cuda"), rows=max(counts + [0]))
        self.check(st, self.m.append(units, rows))

    def fork(self, src, dst):
        st = self.G.pages_fork(self.pg, _i32(src), _i32(dst))
        self.check(st, self.m.fork(src, dst))

    def compact(self, src, keep, idx, dst=None):
        rows = max([len(x) for x in idx] + [0])
        pad = [list(x) + [-5] * (rows - len(x)) for x in idx]
        st = self.G.pages_compact(self.pg, _i32(pad) if rows else None, units=_i32(src),
                                  dst=None if dst is None else _i32(dst), keep=_i32(keep),
                                  counts=_i32([len(x) for x in idx]) if rows else None)
        self.check(st, self.m.compact(src, src if dst is None else dst, keep, idx))

    def free(self, units):
        self.check(self.G.pages_free(self.pg, _i32(units)), self.m.free(units))


@pytest.mark.parametrize("ps,d,dtype", [(16, 64, torch.bfloat16), (64, 128, torch.bfloat16),
                                        (32, 64, torch.float32), (128, 128, torch.float32)])
def test_random_calls(ps, d, dtype):
    rng = random.Random(ps + d)
    p = Pair(9, 5, 26, ps, d, dtype, seed=ps)
    for step in range(60):
        op = rng.choice(["append", "append", "fork", "compact", "compact", "copy", "free"])
        n = rng.randint(1, 4)
        units = [rng.randint(-1, 9) if rng.random() < 0.1 else rng.randrange(9) for _ in range(n)]
        print("step", step, op, units, flush=True)
        held = lambda u: p.m.lens[u] if 0 <= u < 9 else 0  # noqa: E731
        if op == "append":
            p.append(units, [rng.choice([0, 1, rng.randrange(3 * ps)]) for _ in units],
                     rng.choice([torch.bfloat16, torch.float32]), rng.choice([torch.bfloat16, torch.float32]))
        elif op == "fork":
            p.fork(units, [rng.randrange(9) for _ in units])
        elif op == "free":
            p.free(units)
        else:
            keep = [rng.choice([0, held(u), rng.randint(0, held(u) + (rng.random() < 0.1))]) for u in units]
            idx = [[rng.randrange(held(u)) for _ in range(rng.choice([0, 1, rng.randrange(2 * ps)]))]
                   if held(u) else [] for u in units]
            dst = None
            if op == "copy":
                dst = [u if rng.random() < 0.3 else rng.randrange(9) for u in units]
            p.compact(units, keep, idx, dst)


def test_full_pool_and_long_units():
    p = Pair(6, 3, 7, 16, 64, torch.bfloat16)
    p.append([0, 1, 2, 3], [48, 33, 17, 1])     # 3 + 3 pages; the third needs two of one left
    p.append([0, 4], [1, 16])                   # unit 0 is at its table's end
    p.append([5, 1], [1, 15])                   # no page left; unit 1 needs none
    p.fork([0, 1], [2, 3])                      # both are full pages alone: nothing to copy
    p.compact([1], [40], [[]])                  # taken back: its last page is shared now
    p.free([2, 3, 4])
    p.compact([1], [40], [[]])
    p.append([1], [9])


def test_indices_outside_their_unit_give_rows_of_zeros():
    p = Pair(3, 4, 12, 16, 64, torch.float32)
    p.append([0, 1], [30, 20])
    p.compact([0, 1], [17, 3], [[30, 2, -1], [19]])


def test_the_same_unit_twice():
    p = Pair(4, 4, 12, 16, 64, torch.bfloat16)
    p.append([1, 1, 2], [5, 7, 3])
    p.fork([1, 2, 1], [0, 0, 3])                # unit 0 goes to the first
    p.compact([1, 1], [2, 3], [[4], [0]])
    p.compact([2, 2], [1, 2], [[0], [1]], dst=[2, 1])   # read here, written there
    p.free([1, 1, 0, 1])


def test_uniform_rows_default_units_and_lengths_of_zero():
    import paper_2605_31105_amd as G
    p = Pair(5, 4, 20, 32, 128, torch.bfloat16)
    k, v = torch.randn(3, 37, 128), torch.randn(3, 37, 128)
    st = G.pages_append(p.pg, k.cuda(), v.to(torch.bfloat16).cuda())
    rows = [[(k[i, j].bfloat16(), v[i, j].bfloat16()) for j in range(37)] for i in range(3)]
    p.check(st, p.m.append([0, 1, 2], rows))
    idx = torch.stack([torch.randperm(37)[:9].sort().values for _ in range(5)]).int()
    st = G.pages_compact(p.pg, idx.cuda())      # units 3 and 4 are empty: zeros, and said so
    p.check(st, p.m.compact(range(5), range(5), [0] * 5, idx.tolist()))
    st = G.pages_compact(p.pg, keep=_i32([4, 0, 9, 0, 1]))
    p.check(st, p.m.compact(range(5), range(5), [4, 0, 9, 0, 1], [[]] * 5))
    st = G.pages_append(p.pg, torch.empty(2, 0, 128, device="cuda"), torch.empty(2, 0, 128, device="cuda"))
    p.check(st, p.m.append([0, 1], [[], []]))
    st = G.pages_append(p.pg, torch.empty(0, 4, 128, device="cuda"), torch.empty(0, 4, 128, device="cuda"))
    p.check(st, [])
    p.check(G.pages_compact(p.pg), p.m.compact(range(5), range(5), [0] * 5, [[]] * 5))
    p.check(G.pages_free(p.pg), p.m.free(range(5)))


def test_sources_out_of_range():
    import paper_2605_31105_amd as G
    p = Pair(4, 4, 20, 16, 64, torch.bfloat16)
    k, v = p.draw(20, torch.bfloat16, torch.bfloat16)
    starts = torch.tensor([0, 15, -1, 20], device="cuda")
    st = G.pages_append(p.pg, k.cuda(), v.cuda(), starts=starts, rows=6, counts=_i32([9, 6, 1, 0]))
    rows = [[(k[j], v[j]) for j in range(6)], [0] * 6, [0], []]
    p.check(st, p.m.append(range(4), rows, bad=(1, 2)))   # (a count of 9 is taken to 6)


def test_many_entries_and_a_large_pool():
    # more entries than the plan's threads, more pages than one step of its scan, and pages
    # that end up scattered: against the same sums by numpy
    import paper_2605_31105_amd as G
    U, ps, d, pages = 2500, 16, 64, 140000
    pg = G.new_pages(U, 60, pages, ps, d)
    rng = np.random.default_rng(5)
    counts = rng.integers(0, 900, U).astype(np.int32)
    starts = np.zeros(U, np.int64)
    src = torch.arange(1024, device="cuda", dtype=torch.float32)[:, None].expand(1024, d).bfloat16()
    src = src.contiguous()
    st = G.pages_append(pg, src, src, counts=torch.from_numpy(counts).cuda(),
                        starts=torch.from_numpy(starts).cuda(), rows=900)
    need = -(-counts // ps)
    first = np.cumsum(need) - need
    assert not st.any().item() and need.sum() > 65536
    assert np.array_equal(pg.lens.cpu().numpy(), counts)
    table = pg.table.cpu().numpy()
    for u in range(U):
        assert np.array_equal(table[u, :need[u]], first[u] + np.arange(need[u]))
        assert (table[u, need[u]:] == -1).all()
    # every other unit leaves; a second round fills the holes, lowest first, then the end
    gone = torch.arange(0, U, 2, dtype=torch.int32, device="cuda")
    G.pages_free(pg, gone)
    holes = np.concatenate([table[u, :need[u]] for u in range(0, U, 2)])
    rest = np.concatenate([holes, np.arange(need.sum(), pages)])
    half = 900 * np.ones(U // 2, np.int32)
    need2 = -(-half // ps)
    first2 = np.cumsum(need2) - need2
    st = G.pages_append(pg, src, src, units=gone, starts=torch.from_numpy(starts[: U // 2]).cuda(),
                        rows=900).cpu().numpy()
    fits = first2 + need2 <= len(rest)
    assert np.array_equal(st, np.where(fits, 0, 1))
    t2 = pg.table.cpu().numpy()
    for i, u in enumerate(range(0, U, 2)):
        want = rest[first2[i]:first2[i] + need2[i]] if fits[i] else []
        assert np.array_equal(t2[u, :len(want)], want) and (t2[u, len(want):] == -1).all()
    u = 2 * int(np.nonzero(fits)[0][-1])
    rows = pg.k[torch.from_numpy(t2[u, :need2[0]]).long().cuda()].view(-1, d)[:900]
    assert torch.equal(rows, src[:900])
    G.pages_free(pg)
    assert not pg.refs.any().item() and (pg.table == -1).all().item()
    want = torch.full_like(pg.free, -1)
    assert torch.equal(pg.free, want)


def test_captured_calls_and_another_stream():
    # the same round trip captured (three replays, eager calls between them) and on a side
    # stream gives the state of the model
    p = Pair(6, 4, 20, 16, 64, torch.bfloat16)
    G = p.G
    p.append([0, 1], [20, 33])
    k, v = (x.cuda().view(2, 3, 64) for x in p.draw(6, torch.bfloat16, torch.bfloat16))
    rows = [[(k[i, j].cpu(), v[i, j].cpu()) for j in range(3)] for i in range(2)]
    src, dst = _i32([0, 1]), _i32([4, 5])
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = torch.empty(G.pages_workspace_bytes(p.pg, 2), dtype=torch.uint8, device="cuda")

    def calls(stream=None):
        G.pages_fork(p.pg, src, dst, status=st, workspace=ws, stream=stream)
        G.pages_append(p.pg, k, v, units=dst, status=st, workspace=ws, stream=stream)
        G.pages_compact(p.pg, units=dst, keep=_keep, status=st, workspace=ws, stream=stream)
        G.pages_free(p.pg, src, stream=stream, status=st)
        G.pages_fork(p.pg, dst, src, status=st, workspace=ws, stream=stream)
        G.pages_free(p.pg, dst, stream=stream, status=st)

    def model():
        p.m.fork([0, 1], [4, 5])
        p.m.append([4, 5], rows)
        p.m.compact([4, 5], [4, 5], [19, 35], [[], []])
        p.m.free([0, 1])
        p.m.fork([4, 5], [0, 1])
        return p.m.free([4, 5])

    _keep = _i32([19, 35])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls(side)
    side.synchronize()
    p.check(st, model())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        graph.replay()
        p.check(st, model())
        p.append([2], [1])
        p.free([2])


def test_binding_checks():
    import paper_2605_31105_amd as G
    pg = G.new_pages(4, 4, 8, 16, 64)
    k = torch.zeros(2, 3, 64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: G.pages_append(pg, k, k[:, :2].contiguous()),
                 lambda: G.pages_append(pg, k.half(), k.half()),
                 lambda: G.pages_append(pg, k.transpose(0, 1), k.transpose(0, 1)),
                 lambda: G.pages_append(pg, k[0], k[0]),
                 lambda: G.pages_append(pg, k, k, rows=2),
                 lambda: G.pages_append(pg, k, k, units=torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: G.pages_append(pg, k, k, units=torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: G.pages_append(pg, k.cpu(), k.cpu()),
                 lambda: G.pages_append(pg, k[:, :, :32].contiguous(), k[:, :, :32].contiguous()),
                 lambda: G.pages_fork(pg, _i32([0]), _i32([1, 2])),
                 lambda: G.pages_compact(pg, counts=_i32([0])),
                 lambda: G.pages_compact(pg, torch.zeros(2, 3, device="cuda")),
                 lambda: G.Pages(pg.k, pg.v[:4], pg.table, pg.lens, pg.refs, pg.free),
                 lambda: G.Pages(pg.k, pg.v, pg.table, pg.lens, pg.refs[:4], pg.free),
                 lambda: G.Pages(pg.k, pg.v, pg.table.long(), pg.lens, pg.refs, pg.free)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(G.GrkvError):
        G.new_pages(4, 4, 8, 24, 64)
