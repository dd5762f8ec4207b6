"""Attention where its number format shows: weights held to 2^-16 of them, values whose outputs
cancel."""
import pytest

from tests.attention_ref import rows, sink_seen, tree_seen
from tests.test_gpu_attention import BF, F32, _i32, _parents, _pool, _wide_table

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _close(name, o, lse, q, K, V, seen, part=2.0 ** -16):
    """o of bf16 values against float64 rows, for weights held to `part` of them.

    The bounds of float32 values (logits, sums) hold for these too; a weight p_j is off by at most
    part p_j on top (in two bf16 parts: 2^-8 of what the first rounding left, 2^-8), o by part sum
    p_j |v_j|; o is rounded once to bf16, 2^-8 of it."""
    want, wl, tol, tol_lse = rows(q, K, V, seen, False)
    w = torch.where(seen, q.double() @ K.double().t() / q.shape[1] ** 0.5, torch.tensor(-torch.inf, dtype=torch.float64))
    p = torch.exp(w - wl.clamp(min=-1e300)[:, None])
    tol = tol + part * (p @ V.double().abs())
    tol = tol + 2.0 ** -8 * (want.abs() + tol)
    worst = ((o.double() - want).abs() / tol).max().item()
    worst_l = ((lse.double() - wl).abs() / tol_lse).max().item()
    print(name, "o %.2f lse %.2f of the bound" % (worst, worst_l), flush=True)
    assert worst <= 1 and worst_l <= 1, name


@pytest.mark.parametrize("d,ps,group,t,lens,entries,width", [
    (128, 64, 4, 1, [1, 40, 300], 3, 5),             # blocks of 16 rows
    (64, 16, 3, 5, [5, 33, 129, 300], 4, 19),        # a tree
    (128, 64, 4, 2, [600, 570], 2, 10),              # splits that their blocks join
    (128, 16, 2, 9, [9, 100, 260], 70, 17),          # blocks of 32 rows
    (64, 64, 4, 1, [300, 4, 77], 300, 64),           # equal parts
    (128, 64, 5, 6, [6, 300, 64], 300, 40),          # equal parts of 32 rows
])
def test_weights_over_pages_are_held_to_two_parts(d, ps, group, t, lens, entries, width):
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + t)
    pg, K, V = _pool(lens, ps, d, BF, gen)
    if width > pg.table.shape[1]:
        pg = _wide_table(pg, len(lens), width)
    at = [e % len(lens) for e in range(entries)]
    parents, plist = _parents("tree", 1, t, gen)
    q = torch.randn((entries, group, t, d), generator=gen).to(BF)
    o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, parents, units=_i32(at), return_lse=True))
    for e in sorted({*range(len(lens)), entries // 2, entries - 1}):
        for g in range(group):
            _close("entry %d head %d" % (e, g), o[e, g], lse[e, g], q[e, g], K[at[e]], V[at[e]],
                   tree_seen(lens[at[e]], t, plist[0], 0, 0))


@pytest.mark.parametrize("d,group,n,nq,window", [(128, 4, 300, 1, 0), (64, 2, 300, 40, 100), (128, 3, 129, 129, 0)])
def test_weights_of_short_prompts_are_held_to_two_parts(d, group, n, nq, window):
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(n + nq)
    q = torch.randn((2, group, nq, d), generator=gen).to(BF)
    K, V = (torch.randn((2, n, d), generator=gen).to(BF) for _ in range(2))
    o, lse = (x.cpu() for x in G.sink_attention(q.cuda(), K.cuda(), V.cuda(), window, 4, return_lse=True))
    for u in range(2):
        for g in range(group):
            _close("unit %d head %d" % (u, g), o[u, g], lse[u, g], q[u, g], K[u], V[u], sink_seen(n, nq, window, 4))


def test_infinities_that_every_row_sees_stay_infinities():
    # in a tile that is seen whole, past the first of a split, with finite columns beside them
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(21)
    for dtype in (BF, F32):
        pg, K, V = _pool([300, 700], 64, 128, dtype, gen)
        for u, slot in ((0, 70), (1, 500)):
            V[u][slot, 7], V[u][slot, 9] = torch.inf, -torch.inf
            pg.v[int(pg.table[u, slot // 64]), slot % 64] = V[u][slot].cuda()
        q = torch.randn((2, 4, 2, 128), generator=gen).to(dtype)
        o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, units=_i32([0, 1]), return_lse=True))
        assert (o[..., 7] == torch.inf).all() and (o[..., 9] == -torch.inf).all()
        rest = [c for c in range(128) if c not in (7, 9)]
        for u, n in enumerate((300, 700)):
            seen = tree_seen(n, 2, [-1, 0], 0, 0)
            for g in range(4):
                want, wl, tol, _ = rows(q[u, g], K[u], torch.nan_to_num(V[u].float(), 0, 0, 0), seen, dtype == BF)
                assert ((o[u, g].double() - want).abs() <= tol)[:, rest].all()
