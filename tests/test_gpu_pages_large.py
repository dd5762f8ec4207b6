"""The calls on pages at their limits: bounds on the rows near 2^31, pools of many units, many
entries."""
import pytest

from tests.test_gpu_pages import Pair, _i32

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_bounds_on_the_rows_near_two_to_the_31():
    # entries * (rows + page size) just under 2^31, counts of a few rows, a prefix of some pages:
    # rows past a unit's last are none, whatever first slot they would be added to
    p = Pair(3, 6, 30, 16, 64, torch.bfloat16)
    G = p.G
    p.append([0, 1, 2], [70, 40, 33])
    most = (1 << 31) - 1 - 16
    starts = torch.zeros(1, dtype=torch.int64, device="cuda")
    st = G.pages_compact(p.pg, _i32([69, 3, 50]), units=_i32([0]), keep=_i32([64]), counts=_i32([3]),
                         starts=starts, rows=most)
    p.check(st, p.m.compact([0], [0], [64], [[69, 3, 50]]))
    st = G.pages_compact(p.pg, _i32([0]), units=_i32([1]), keep=_i32([41]), counts=_i32([1]),
                         starts=starts, rows=most)                       # refused: more than it holds
    p.check(st, p.m.compact([1], [1], [41], [[0]]))
    half = ((1 << 31) - 1) // 2 - 16
    k, v = p.draw(9, torch.bfloat16, torch.bfloat16)
    st = G.pages_append(p.pg, k.cuda(), v.cuda(), units=_i32([2, 0]), counts=_i32([4, 5]),
                        starts=torch.tensor([5, 0], device="cuda"), rows=half)
    p.check(st, p.m.append([2, 0], [[(k[j], v[j]) for j in range(5, 9)], [(k[j], v[j]) for j in range(5)]]))


class _Filled:
    """The calls on pages, each with a workspace of given bytes."""

    def __init__(self, G, pg, fill, most):
        self.G, self.fill = G, fill
        self.ws = torch.empty(G.pages_workspace_bytes(pg, most), dtype=torch.uint8, device="cuda")

    def __getattr__(self, name):
        call = getattr(self.G, name)
        if name not in ("pages_append", "pages_fork", "pages_compact"):
            return call

        def filled(*args, **kw):
            self.ws.fill_(self.fill)
            return call(*args, workspace=self.ws, **kw)
        return filled


@pytest.mark.parametrize("fill", [0, 255, 3])
def test_pools_of_more_units_than_fit_the_plan(fill):
    # owners in the workspace, which holds anything before: sources named twice, destinations
    # named twice, units read and written, units outside, by more entries than a block has threads
    import random
    rng = random.Random(fill)
    U = 10000
    p = Pair(U, 4, 9000, 16, 64, torch.bfloat16, seed=fill)
    p.G = _Filled(p.G, p.pg, fill, 2000)
    first = rng.sample(range(U), 1500)
    p.append(first, [rng.choice([0, 1, 15, 16, 17, rng.randrange(60)]) for _ in first])
    src = [rng.choice(first) for _ in range(1300)]
    dst = [rng.choice([rng.randrange(U), U - 1 - k, rng.choice(first)]) for k in range(1300)]
    src[7], dst[9], src[1200], dst[1201] = U, -1, dst[3], dst[2]
    p.fork(src, dst)
    held = p.m.lens
    units = [rng.choice(first) if k % 3 else rng.randrange(U) for k in range(1200)]
    keep = [rng.randint(0, held[u]) for u in units]
    idx = [[rng.randrange(held[u]) for _ in range(rng.randrange(20))] if held[u] else [] for u in units]
    p.compact(units, keep, idx)                                  # in place, many of them twice
    held = p.m.lens
    units = [rng.choice(first) for _ in range(1100)]
    to = [u if k % 4 == 0 else rng.randrange(U) for k, u in enumerate(units)]
    keep = [rng.randint(0, held[u]) for u in units]
    idx = [[rng.randrange(held[u]) for _ in range(rng.randrange(12))] if held[u] else [] for u in units]
    p.compact(units, keep, idx, dst=to)
    units = rng.sample(range(U), 1100)
    p.compact(units, [p.m.lens[u] // 2 for u in units], [[]] * 1100)   # taken back
    p.append([5, 5, U, -3, 9999], [3, 4, 1, 1, 40])
    p.free([rng.randrange(U) for _ in range(1500)])


def test_long_rows_of_many_entries():
    # more than 256 rows an entry and 512 entries or more: an entry is one block's still
    import random
    rng = random.Random(6)
    p = Pair(600, 24, 600 * 24, 16, 64, torch.bfloat16)
    p.append(list(range(520)), [320 + k % 40 for k in range(520)])
    units = rng.sample(range(520), 520)
    keep = [rng.choice([0, 5, 16, 33]) for _ in units]
    idx = [[rng.randrange(320) for _ in range(257 + k % 50)] for k in range(520)]
    p.compact(units, keep, idx)
    p.compact(units[:100], [0] * 100, [[rng.randrange(257) for _ in range(300)] for _ in range(100)])   # fewer: spread


def test_a_unit_forked_to_itself_stays():
    p = Pair(4, 4, 12, 16, 64, torch.bfloat16)
    p.append([0, 1, 2], [20, 32, 0])
    p.fork([1], [3])                            # unit 1's pages are shared
    p.fork([0, 1, 2], [0, 1, 2])
    assert p.m.lens == [20, 32, 0, 32]
    p.fork([0, 0], [0, 2])                      # read by the second entry, the first's own
    assert p.m.lens == [20, 32, 0, 32]


def test_a_pool_made_on_another_stream_owns_its_memory_there():
    # memory that the current stream has let go of but still writes is not the new pool's
    import paper_2605_31105_amd as G
    x = torch.empty((1024, 4096), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    x.fill_(7)
    del x
    pg = G.new_pages(1024, 4096, 64, 16, 64, stream=side)
    torch.cuda.synchronize()
    assert (pg.table == -1).all() and not pg.lens.any() and (pg.free == -1).all()
    with torch.cuda.stream(side):
        assert not G.pages_append(pg, *(torch.ones(3, 5, 64, device="cuda") for _ in range(2))).any()
    side.synchronize()
    assert pg.lens[:4].tolist() == [5, 5, 5, 0]
