"""Attention where its number format shows: weights held to 2^-15 of them, values whose outputs
cancel, values near a float's largest."""
import pytest

from tests.attention_ref import check, rows, sink_seen, tree_seen
from tests.test_gpu_attention import BF, F32, _i32, _parents, _pool, _wide_table

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _close(name, o, lse, q, K, V, seen, part=2.0 ** -15 + 2.0 ** -18):
    """o of bf16 values against float64 rows, for weights held to `part` of them.

    The bounds of float32 values (logits, sums) hold for these too; a weight p_j is off by at most
    part p_j on top (in two bf16 parts: the upper bits leave less than 2^-7 of it, whose rounding is
    off by 2^-8 of that, and 2^-18 of it is added), o by part sum p_j |v_j|; o is rounded once to
    bf16, 2^-8 of it."""
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


def _ramp(q, K, V, lo, hi):
    """Logits that rise along the keys from lo to hi (log2), values of 1e36 and random signs."""
    d, n = K.shape[-1], K.shape[-2]
    q[..., :2] = torch.tensor([8.0, 0.0])
    K[..., 0] = torch.linspace(lo, hi, n) * d ** 0.5 / 1.4426950408889634 / 8
    K[..., 2:] *= 0.1
    V *= 1e36


@pytest.mark.parametrize("dtype,d,group,t,lens,entries,width", [
    (BF, 128, 4, 1, [300, 40], 2, 5), (BF, 64, 2, 3, [900, 33], 2, 20), (F32, 128, 4, 2, [500], 1, 9),
    (F32, 64, 1, 1, [100, 17], 2, 9), (BF, 128, 2, 9, [300, 1500], 2, 900), (BF, 64, 4, 2, [900, 5], 300, 60),
    (BF, 128, 4, 8, [300, 900], 70, 20), (BF, 128, 5, 16, [900, 70], 300, 20), (BF, 64, 40, 4, [600, 5], 300, 20),
])
def test_large_values_under_growing_logits(dtype, d, group, t, lens, entries, width):
    # weights against an early, low reference must not carry finite values past a float's range:
    # logits that rise by 39 (log2) under values of 1e36, whose outputs are of that size
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(t)
    pg, K, V = _pool(lens, 64, d, dtype, gen)
    q = torch.randn((entries, group, t, d), generator=gen)
    for u, n in enumerate(lens):
        K[u], V[u] = K[u].float(), V[u].float()
        _ramp(q, K[u], V[u], -19.5, 19.5)
        K[u], V[u] = K[u].to(dtype), V[u].to(dtype)
        slot = torch.arange(n, device="cuda")
        pg.k[pg.table[u, slot // 64].long(), slot % 64] = K[u].cuda()
        pg.v[pg.table[u, slot // 64].long(), slot % 64] = V[u].cuda()
    q = q.to(dtype)
    if width > pg.table.shape[1]:
        pg = _wide_table(pg, len(lens), width)
    at = [e % len(lens) for e in range(entries)]
    if group * t > 64:   # (the wide kernel's)
        assert dtype == BF and entries * group * t * width * 64 > 1 << 20
    o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, units=_i32(at), return_lse=True))
    for e in (*range(len(lens)), entries - 1):
        u = at[e]
        seen = tree_seen(lens[u], t, list(range(-1, t - 1)), 0, 0)
        for g in range(0, group, 3):
            check("entry %d head %d" % (e, g), o[e, g], lse[e, g], q[e, g], K[u], V[u], seen)


@pytest.mark.parametrize("dtype,d,group,n,nq", [(BF, 128, 2, 1100, 1100), (BF, 64, 4, 800, 800), (F32, 64, 2, 300, 100),
                                                (BF, 128, 3, 200, 9)])
def test_large_values_of_a_prompt_under_growing_logits(dtype, d, group, n, nq):
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(n)
    q = torch.randn((1, group, nq, d), generator=gen)
    K, V = (torch.randn((1, n, d), generator=gen) for _ in range(2))
    _ramp(q, K, V, -19.5, 19.5)
    q, K, V = q.to(dtype), K.to(dtype), V.to(dtype)
    assert nq < 800 or group * nq * n > 1 << 20   # (the long ones are the wide kernel's)
    o, lse = (x.cpu() for x in G.sink_attention(q.cuda(), K.cuda(), V.cuda(), 0, return_lse=True))
    for g in range(group):
        check("head %d" % g, o[0, g], lse[0, g], q[0, g], K[0], V[0], sink_seen(n, nq, 0, 0))


def test_values_at_the_types_largest():
    # one key far above the others, whose value is the largest finite one
    import paper_2605_31105_amd as G
    for dtype in (BF, F32):
        K, V = torch.zeros(1, 300, 64, dtype=dtype), torch.full((1, 300, 64), -1.0, dtype=dtype)
        K[0, 200, 0] = 1000.0
        V[0, 200] = torch.finfo(dtype).max
        V[0, 5] = torch.finfo(dtype).min
        q = torch.zeros(1, 2, 1, 64, dtype=dtype)
        q[..., 0] = 8.0
        o = G.sink_attention(q.cuda(), K.cuda(), V.cuda(), 0).cpu()
        assert (o == torch.finfo(dtype).max).all(), o


def test_large_values_summed_over_splits():
    # the kernel of many rows, 4 tiles and more a split: a peak of 2^15 over the first tiles'
    # logits in every fourth tile, whose parts are finite while their sum against those logits
    # is not; o is the peaks' value
    import paper_2605_31105_amd as G
    n, d, group = 65536, 64, 40
    K, V = torch.zeros((n, d)), torch.zeros((n, d))
    peak = torch.arange(n // 256) * 256 + 3 * 64 + 17
    K[peak, 0] = 15 * d ** 0.5 / 1.4426950408889634 / 8
    V[peak] = 2.0 ** 110
    V[peak, 1] = -(2.0 ** 110)
    pg = G.new_pages(1, n // 64, n // 64, 64, d)
    K, V = K.to(BF), V.to(BF)
    assert not G.pages_append(pg, K[None].cuda(), V[None].cuda()).any().item()
    q = torch.zeros((1, group, 2, d), dtype=BF)
    q[..., 0] = 8.0
    o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, return_lse=True))
    seen = tree_seen(n, 2, [-1, 0], 0, 0)
    for g in (0, group - 1):
        check("head %d" % g, o[0, g], lse[0, g], q[0, g], K, V, seen)


@pytest.mark.parametrize("dtype,d,group,t", [(BF, 128, 1, 1), (F32, 64, 1, 1), (BF, 64, 5, 6), (BF, 128, 40, 2), (BF, 64, 40, 2)])
def test_logits_past_a_floats_step(dtype, d, group, t):
    # logits of 10^10, a step of which is many powers of two: a row's largest still has a weight
    # (o is that key's value), whichever way the reference was rounded.  A unit's rows are alike.
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + group)
    n, top, E = 500, 211, 40
    pg, K, V = _pool([n], 64, d, dtype, gen)
    pg = _wide_table(pg, 1, 12)
    assert group * t <= 64 or E * group * t * 12 * 64 > 1 << 20
    sign = torch.randint(0, 2, (d,), generator=gen) * 2.0 - 1
    q = (sign * (20000 + 20000 * torch.rand((E, 1, 1, d), generator=gen))).expand(E, group, t, d).to(dtype).contiguous()
    K[0] = (K[0].float() * 1000).to(dtype)
    K[0][top] = (sign * 30000).to(dtype)
    slot = torch.arange(n, device="cuda")
    pg.k[pg.table[0, slot // 64].long(), slot % 64] = K[0].cuda()
    o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, units=_i32([0] * E), return_lse=True))
    logit = (q.double() @ K[0][top].double()) / d ** 0.5
    assert ((lse.double() - logit).abs() <= 2.0 ** -18 * logit).all()
    # o = (w v) (1 / l) with l = w, which need not be a power of two: the product, the reciprocal (one
    # step, 2^-23) and their product are off by at most 2^-24 + 2^-23 + 2^-24 = 2^-22 together; the
    # rounding to bf16 takes that, and the weights' 2^-15, back to v
    v = V[0][top].expand(E, group, t, d)
    off = (o.double() - v.double()).abs()
    assert (off <= (0.0 if dtype == BF else 2.0 ** -22) * v.double().abs()).all()
