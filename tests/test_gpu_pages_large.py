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
