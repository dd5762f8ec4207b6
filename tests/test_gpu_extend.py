"""The units of a step grown (pages_extend) against the definition in plain Python, bit for bit."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

FULL, LENGTH, UNIT, RANGE = 1, 2, 3, 4


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Model:
    """A pool's tables, one page at a time."""

    def __init__(self, units, width, pages, ps):
        self.ps, self.width, self.pages = ps, width, pages
        self.table, self.lens, self.refs = [[] for _ in range(units)], [0] * units, [0] * pages

    def extend(self, counts, tokens, units, seen):
        """starts, positions, slots, status; units [B][H]."""
        B, H = len(counts), len(units[0])
        counts = [max(c, 0) for c in counts]
        total, starts, status = 0, [], []
        named = {}
        for b in range(B):
            for u in units[b]:
                named.setdefault(u, []).append(b)
        first_use = set()
        ok_units = [u for row in units for u in row]
        firsts = []
        for b in range(B):
            code = 0
            at = total
            total += counts[b]
            starts.append(min(at, tokens))
            u0 = units[b][0]
            first = seen[b] if seen is not None else (self.lens[u0] if 0 <= u0 < len(self.lens) else 0)
            firsts.append(first)
            if counts[b] and (total > tokens or first < 0 or first > 2 ** 31 - 1 - counts[b]):
                code = RANGE
            for u in units[b]:
                if not 0 <= u < len(self.lens) or u in first_use:
                    code = max(code, UNIT)
                    continue
                first_use.add(u)
                if self.lens[u] + counts[b] > self.width * self.ps:
                    code = max(code, LENGTH)
            status.append(code)
        starts.append(min(total, tokens))
        assert len(ok_units) == B * H
        # pages in order; a sequence whose pages pass the free ones is refused, and all behind it
        free = [p for p, r in enumerate(self.refs) if r == 0]
        need = {}
        for b in range(B):
            need[b] = [0] * H if status[b] else [
                -(-(self.lens[u] + counts[b]) // self.ps) + -self.lens[u] // self.ps for u in units[b]]
        at = 0
        positions, slots = [-(1 << 31)] * tokens, [[-1] * H for _ in range(tokens)]
        for b in range(B):
            mine = sum(need[b])
            at += mine
            if status[b] == 0 and mine and at > len(free):
                status[b] = FULL
            if status[b]:
                continue
            take = at - mine
            for h, u in enumerate(units[b]):
                for _ in range(need[b][h]):
                    self.table[u].append(free[take])
                    self.refs[free[take]] = 1
                    take += 1
                for i in range(counts[b]):
                    s = self.lens[u] + i
                    slots[starts[b] + i][h] = self.table[u][s // self.ps] * self.ps + s % self.ps
                self.lens[u] += counts[b]
            for i in range(counts[b]):
                positions[starts[b] + i] = firsts[b] + i
        return starts, positions, slots, status

    def free_words(self):
        words = [0] * (-(-self.pages // 32))
        for p, r in enumerate(self.refs):
            words[p // 32] |= (r == 0) << (p % 32)
        return [w - (1 << 32) if w >> 31 else w for w in words]

    def same(self, pg):
        table = [t + [-1] * (self.width - len(t)) for t in self.table]
        assert pg.lens.tolist() == self.lens
        assert pg.table.tolist() == table
        assert pg.refs.tolist() == self.refs
        assert pg.free.tolist() == self.free_words()


def _both(pg, m, counts, tokens, units=None, heads=None, seen=None, **kw):
    import paper_2605_31105_amd as G
    B = len(counts)
    rows = units if units is not None else [[b * heads + h for h in range(heads)] for b in range(B)]
    got = G.pages_extend(pg, _i32(counts), tokens, heads=heads if units is None else None,
                         units=None if units is None else _i32(units), seen=None if seen is None else _i32(seen), **kw)
    starts, positions, slots, status = m.extend(counts, tokens, rows, seen)
    assert got.status.tolist() == status
    assert got.starts.tolist() == starts
    assert got.positions.tolist() == positions
    assert got.slots.tolist() == slots
    m.same(pg)
    return status


@pytest.mark.parametrize("seed", range(8))
def test_random_steps(seed):
    import paper_2605_31105_amd as G
    rng = random.Random(seed)
    ps, U = rng.choice([16, 32, 64]), rng.choice([7, 24, 60])
    width = rng.choice([2, 5, 40])
    pages = rng.choice([U, 3 * U, U * width // 2 + 1, 2000])
    pg, m = G.new_pages(U, width, pages, ps, 64), Model(U, width, pages, ps)
    seen_codes = set()
    for turn in range(25):
        H = rng.choice([1, 2, 3, 6])
        B = rng.randint(1, max(1, U // H))
        listed = rng.random() < 0.6
        units = None
        if listed:
            flat = rng.sample(range(U), min(U, B * H))
            B = max(1, len(flat) // H)
            flat = (flat + [0] * H)[:B * H]
            units = [flat[b * H:b * H + H] for b in range(B)]
            if rng.random() < 0.3:
                units[rng.randrange(B)][rng.randrange(H)] = rng.choice([-1, U, 1 << 30, units[0][0]])
        counts = [rng.choice([0, 1, 1, rng.randint(0, 3 * ps), -3]) for _ in range(B)]
        total = sum(max(c, 0) for c in counts)
        tokens = max(0, total + rng.choice([0, 0, 5, -1, -total // 2]))
        seen = [rng.choice([0, 5, 1 << 20, 2 ** 31 - 2, -1]) for _ in range(B)] if rng.random() < 0.5 else None
        seen_codes |= set(_both(pg, m, counts, tokens, units, H, seen))
        if rng.random() < 0.2:
            drop = rng.sample(range(U), rng.randint(1, U))
            G.pages_free(pg, _i32(drop))
            for u in drop:
                for p in m.table[u]:
                    m.refs[p] = 0
                m.table[u], m.lens[u] = [], 0
    print(seed, "codes", sorted(seen_codes), flush=True)


def test_every_refusal_by_hand():
    import paper_2605_31105_amd as G
    pg, m = G.new_pages(6, 2, 5, 16, 64), Model(6, 2, 5, 16)
    assert _both(pg, m, [16, 17], 40, [[0, 1], [2, 3]]) == [0, FULL]      # 2 pages, then 4 of 3
    assert _both(pg, m, [17, 1], 40, [[0, 1], [4, 5]]) == [LENGTH, 0]     # 33 rows of 32
    assert _both(pg, m, [1, 0, 1], 9, [[2, 2], [0, 3], [3, 6]]) == [UNIT, 0, UNIT]
    assert _both(pg, m, [2, 0, 1], 2, [[2, 3], [0, 1], [4, 5]]) == [FULL, 0, RANGE]
    assert _both(pg, m, [3, 3], 4, [[4, 5], [2, 3]]) == [0, RANGE]
    assert _both(pg, m, [1, 1], 2, [[4, 5], [2, 3]], seen=[2 ** 31 - 2, 2 ** 31 - 1]) == [0, RANGE]
    assert _both(pg, m, [0, 0], 0, [[4, 5], [2, 3]]) == [0, 0]


@pytest.mark.parametrize("U,H,B", [(9000, 3, 1500), (9000, 1, 1), (20000, 250, 40)])
def test_many_units_and_sequences(U, H, B):
    # more units than the plan's LDS holds, more sequences and entries than it has threads
    import paper_2605_31105_amd as G
    rng = random.Random(U + B)
    ps, width, pages = 16, 6, 2 * U + 7
    pg, m = G.new_pages(U, width, pages, ps, 64), Model(U, width, pages, ps)
    for turn in range(2):
        counts = [rng.choice([0, 1, rng.randint(1, 40)]) for _ in range(B)]
        flat = rng.sample(range(U), B * H)
        units = [flat[b * H:b * H + H] for b in range(B)]
        _both(pg, m, counts, sum(counts) + turn, units)
    _both(pg, m, counts, sum(counts), None, H)
    # a unit that is not there, one named twice, rows past the step's and, in the end, no pages left
    units[B // 2][H - 1], units[B - 1][0] = U, units[0][0]
    bad = _both(pg, m, counts, sum(counts) - 1, units)
    assert bad[B // 2] in (UNIT, RANGE) and bad[B - 1] in (UNIT, RANGE)   # (the largest of its codes)
    for _ in range(4):
        more = [max(c, 12) for c in counts]
        codes = _both(pg, m, more, sum(more), None, H)
    print(U, H, B, "codes", sorted(set(codes)), flush=True)


def test_a_units_matrix_with_strides_and_a_step_used_again():
    # a layer's columns of a model's units; the outputs of the call before written again
    import paper_2605_31105_amd as G
    B, L, H = 3, 4, 2
    pg, m = G.new_pages(B * L * H, 4, 200, 16, 64), Model(B * L * H, 4, 200, 16)
    every = torch.arange(B * L * H, dtype=torch.int32, device="cuda").view(B, L, H)
    out = None
    for counts in ([5, 0, 17], [1, 1, 1], [0, 30, 2]):
        for layer in range(L):
            got = G.pages_extend(pg, _i32(counts), 33, units=every[:, layer], out=out)
            want = m.extend(counts, 33, every[:, layer].tolist(), None)
            assert [got.starts.tolist(), got.positions.tolist(), got.slots.tolist(), got.status.tolist()] == list(want)
            assert out is None or got is out
            out = got
    m.same(pg)
    whole = G.pages_extend(pg, _i32([1, 2, 3]), 6, units=every.view(B, L * H))
    want = m.extend([1, 2, 3], 6, every.view(B, L * H).tolist(), None)
    assert whole.slots.tolist() == want[2] and whole.positions.tolist() == want[1]


def test_captured_steps_and_another_stream():
    # every replay of a captured step grows the units again
    import paper_2605_31105_amd as G
    B, H, tokens = 4, 3, 12
    pg, m = G.new_pages(B * H, 8, 300, 16, 64), Model(B * H, 8, 300, 16)
    counts, seen = _i32([1, 3, 0, 7]), _i32([100, 5, 9, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = G.pages_extend(pg, counts, tokens, heads=H, seen=seen, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    rows = [[b * H + h for h in range(H)] for b in range(B)]
    assert out.slots.tolist() == m.extend([1, 3, 0, 7], tokens, rows, [100, 5, 9, 0])[2]
    ws = torch.empty(G.pages_extend_workspace_bytes(pg, B, H, tokens), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.pages_extend(pg, counts, tokens, heads=H, seen=seen, out=out, workspace=ws)
    for turn in range(4):
        c = [turn, 2, 5 - turn, 1]
        counts.copy_(_i32(c))
        ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        want = m.extend(c, tokens, rows, [100, 5, 9, 0])
        assert [out.starts.tolist(), out.positions.tolist(), out.slots.tolist(), out.status.tolist()] == list(want)
        m.same(pg)


def test_no_sequences_and_binding_checks():
    import paper_2605_31105_amd as G
    pg = G.new_pages(4, 2, 9, 16, 64)
    none = G.pages_extend(pg, _i32([]), 3, heads=2)
    assert none.starts.tolist() == [0] and none.slots.tolist() == [[-1, -1]] * 3
    assert none.positions.tolist() == [G.NO_POSITION] * 3 and none.status.tolist() == []
    c = _i32([1, 1])
    for call in (lambda: G.pages_extend(pg, c, 2), lambda: G.pages_extend(pg, c.long(), 2, heads=2),
                 lambda: G.pages_extend(pg, c.cpu(), 2, heads=2), lambda: G.pages_extend(pg, c, -1, heads=2),
                 lambda: G.pages_extend(pg, c, 2, units=c), lambda: G.pages_extend(pg, c, 2, heads=3, units=_i32([[0, 1], [2, 3]])),
                 lambda: G.pages_extend(pg, c, 2, heads=2, seen=_i32([1])), lambda: G.pages_extend(pg, c, 1 << 32, heads=2),
                 lambda: G.pages_extend(pg, c, 3, heads=2, out=none), lambda: G.pages_extend(pg, c, 2, units=_i32([[0, 1]])),
                 lambda: G.pages_extend(pg, c, 2, units=_i32([[0, 1], [2, 3]]).t())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: G.pages_extend(pg, c, 2, units=_i32([[0, 1]]).expand(2, 2)), lambda: G.pages_extend(pg, c, 1 << 30, heads=2, out=G.Step(
            none.starts, none.positions, none.slots, none.status))):
        with pytest.raises((G.GrkvError, ValueError)):
            call()
    assert pg.lens.tolist() == [0] * 4
