"""Attention of a step's new tokens (chunk_attention) against float64 rows, within the bounds of
tests/attention_ref.py."""
import math

import pytest

from tests.attention_ref import check, sink_seen
from tests.test_gpu_attention import BF, F32, _i32, _pool
from tests.test_gpu_attention_values import _close, _ramp

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _run(name, lens, counts, H, group, ps, d, dtype, window=0, n_sink=0, pad=0, longest=None, heads=None):
    """A call on units of these lengths (new tokens included), checked row by row; lens [B][H]."""
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + ps)
    flat = [n for row in lens for n in row]
    pg, K, V = _pool(flat, ps, d, dtype, gen)
    B, T = len(counts), sum(counts) + pad
    q = torch.randn((T, H * group, d), generator=gen).to(dtype)
    starts = [sum(counts[:b]) for b in range(B + 1)]
    o = torch.full(q.shape, 5.0, dtype=dtype, device="cuda")
    lse = torch.full(q.shape[:2], 6.0, device="cuda")
    G.chunk_attention(q.cuda(), pg, _i32(starts), heads=H, longest=longest, window=window, n_sink=n_sink,
                      out=o, lse=lse)
    torch.cuda.synchronize()
    o, lse = o.cpu(), lse.cpu()
    assert (o[starts[-1]:] == 5).all() and (lse[starts[-1]:] == 6).all()
    for b, c in enumerate(counts):
        m = min(c, longest) if longest else c
        at = slice(starts[b], starts[b] + m)
        assert (o[starts[b] + m:starts[b + 1]] == 5).all() and (lse[starts[b] + m:starts[b + 1]] == 6).all()
        for h in range(H) if heads is None else heads:
            n, u = lens[b][h], b * H + h
            seen = sink_seen(n, m, window, n_sink)
            for g in {0, group - 1}:
                x = h * group + g
                check("%s seq %d (%d of %d) head %d" % (name, b, m, n, x), o[at, x], lse[at, x], q[at, x], K[u], V[u],
                      seen)
    return o, lse


CASES = [
    # dtype, d, page, group, new tokens, lengths before them (per sequence; units differ by 3), window, sinks
    (BF, 128, 64, 4, [1, 1, 1], [0, 63, 2000], 0, 0), (BF, 64, 16, 1, [5, 1, 40], [0, 300, 17], 0, 0),
    (BF, 128, 64, 4, [300, 1, 0, 33, 5], [500, 900, 10, 0, 64], 0, 0), (BF, 128, 16, 5, [129, 2], [77, 1000], 0, 0),
    (BF, 64, 256, 8, [16, 17, 2, 3], [1000, 0, 5, 64], 0, 0), (BF, 128, 1024, 3, [600], [700], 0, 0),
    (BF, 64, 32, 7, [100, 1, 9], [900, 900, 900], 100, 4), (BF, 128, 64, 4, [200, 1], [300, 2500], 64, 70),
    (BF, 128, 64, 16, [1, 2, 40], [100, 100, 100], 1, 0), (BF, 64, 64, 33, [4, 1], [60, 700], 37, 300),
    (F32, 128, 32, 3, [5, 100, 0, 1], [100, 40, 7, 900], 0, 0), (F32, 64, 16, 4, [33, 1, 1], [0, 16, 500], 0, 0),
    (F32, 64, 64, 5, [50, 3], [300, 1000], 60, 5), (F32, 128, 16, 17, [3, 1], [100, 31], 0, 0),
    (BF, 128, 64, 1, [129, 127, 128, 1], [0, 1, 0, 0], 0, 0), (BF, 64, 16, 2, [0, 0, 64, 0, 65, 0], [5] * 6, 0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-d%d-p%d-g%d-c%s-w%d" % (
    "bf16" if c[0] == BF else "f32", c[1], c[2], c[3], "_".join(map(str, c[4])), c[6]))
def test_chunk_attention(case):
    dtype, d, ps, group, counts, before, window, n_sink = case
    H = 2
    lens = [[max(b + 3 * h, 0) + c for h in range(H)] for b, c in zip(before, counts)]
    _run("case", lens, counts, H, group, ps, d, dtype, window, n_sink, pad=5)


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (64, F32)])
def test_units_shorter_than_their_new_tokens_and_bad_units(d, dtype):
    # the first queries see nothing; units outside the pool see nothing; longest cuts
    import paper_2605_31105_amd as G
    _run("short", [[3, 0], [40, 100], [0, 200]], [10, 90, 150], 2, 2, 16, d, dtype)
    _run("window", [[3, 0], [40, 100], [0, 200]], [10, 90, 150], 2, 2, 16, d, dtype, window=20, n_sink=3)
    _run("cut", [[30, 30], [300, 100]], [30, 90], 2, 3, 16, d, dtype, longest=7, pad=1)
    gen = torch.Generator().manual_seed(1)
    pg, K, V = _pool([50, 60], 16, d, dtype, gen)
    q = torch.randn((6, 4, d), generator=gen).to(dtype).cuda()
    o, lse = G.chunk_attention(q, pg, _i32([0, 4, 6]), units=_i32([[-1, 1], [0, 99]]), return_lse=True)
    for rows, heads in ((slice(0, 4), slice(0, 2)), (slice(4, 6), slice(2, 4))):
        assert (o[rows, heads] == 0).all() and torch.isneginf(lse[rows, heads]).all()
    check("unit 1", o[:4, 2].cpu(), lse[:4, 2].cpu(), q[:4, 2].cpu(), K[1], V[1], sink_seen(60, 4, 0, 0))
    check("unit 0", o[4:, 1].cpu(), lse[4:, 1].cpu(), q[4:, 1].cpu(), K[0], V[0], sink_seen(50, 2, 0, 0))


@pytest.mark.parametrize("d", [64, 128])
def test_long_units_cut_into_many_parts(d):
    # single tokens over long keys, beside chunks: parts that begin and end inside units
    _run("long", [[20001, 5], [300, 9000], [1, 1], [4000, 7777]], [1, 3, 1, 1], 2, 4, 64, d, BF)
    _run("beside", [[20500, 800], [300, 9000]], [500, 1], 2, 4, 64, d, BF, heads=[0, 1])
    _run("one", [[30000]], [1], 1, 8, 128, d, BF)
    _run("wide", [[6000]], [40], 1, 4, 128, d, BF)


def test_many_sequences_of_one_token():
    lens = [[1 + (37 * b + 11 * h) % 700 for h in range(3)] for b in range(300)]
    _run("many", lens, [1] * 300, 3, 4, 16, 64, BF, heads=[1])


def test_more_sequences_than_a_block_holds_starts_of():
    lens = [[1 + (7 * b) % 40] for b in range(1500)]
    _run("1500", lens, [1 if b % 7 else 0 for b in range(1500)], 1, 2, 16, 64, BF)
    counts = [1 + (b % 600 == 5) * 70 for b in range(1200)]
    _run("1200", [[c + (3 * b) % 20] for b, c in enumerate(counts)], counts, 1, 2, 16, 64, F32)


def test_many_short_jobs_and_idle_sequences():
    counts = [(b * 7) % 23 if b % 3 else 0 for b in range(150)]
    lens = [[c + (13 * b) % 90 for _ in range(2)] for b, c in enumerate(counts)]
    _run("short", lens, counts, 2, 3, 16, 64, BF, pad=9)


@pytest.mark.parametrize("dtype,group,counts", [(BF, 2, [6]), (BF, 16, [12, 1]), (F32, 2, [6]), (BF, 4, [100])])
def test_what_a_query_does_not_see_never_reaches_it(dtype, group, counts):
    # NaN and infinities among later keys and values, and in the slots behind a unit
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(3)
    n, d = 70 + counts[0], 64
    pg, K, V = _pool([n] + [40] * (len(counts) - 1), 16, d, dtype, gen)
    bad = n - 3
    q = torch.randn((sum(counts), group, d), generator=gen).to(dtype)
    starts = _i32([0] + [sum(counts[:b + 1]) for b in range(len(counts))])
    for value in (math.nan, math.inf, -math.inf):
        for x in (pg.k, pg.v):
            x[pg.table[0, bad // 16].long(), bad % 16] = value
        o, lse = (x.cpu() for x in G.chunk_attention(q.cuda(), pg, starts, heads=1, return_lse=True))
        c = counts[0]
        before = c - 3                     # queries that lie before the bad slot
        seen = sink_seen(n, c, 0, 0)[:before, :bad]
        for g in {0, group - 1}:
            check("%s head %d" % (value, g), o[:before, g], lse[:before, g], q[:before, g], K[0][:bad], V[0][:bad], seen)
        assert not torch.isfinite(o[before:c]).all()
        assert torch.isfinite(o[c:]).all()


def test_large_logits_and_values():
    # growing logits move the reference; weights of zero beside logits past 2^30; values near the largest float
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(5)
    d, n, c = 64, 400, 40
    for group in (1, 8):
        pg, K, V = _pool([n], 16, d, BF, gen)
        for j in range(n):
            K[0][j] = 0
            K[0][j, 0] = j / 4
        pg.k.view(-1, d)[(pg.table[0].long()[torch.arange(n) // 16] * 16).cpu() + torch.arange(n) % 16] = K[0].cuda()
        q = torch.zeros((c, group, d), dtype=BF)
        q[..., 0] = torch.linspace(-20, 20, c)[:, None].to(BF)
        o, lse = (x.cpu() for x in G.chunk_attention(q.cuda(), pg, _i32([0, c]), heads=1, return_lse=True))
        for g in {0, group - 1}:
            check("growing", o[:, g], lse[:, g], q[:, g], K[0], V[0], sink_seen(n, c, 0, 0))


@pytest.mark.parametrize("d,group,counts,lens", [
    (128, 4, [1, 3, 4], [300, 40, 2000]), (64, 3, [5, 1, 0], [129, 33, 7]), (128, 4, [1] * 90, [20 + 31 * b for b in range(90)]),
    (64, 16, [1, 1], [9000, 20]), (128, 4, [5, 8, 1, 6], [300, 40, 9000, 6]), (64, 3, [10, 9], [129, 33]),
    (128, 7, [4, 3] * 40, [20 + 31 * b for b in range(80)])])
def test_weights_of_few_rows_are_held_to_two_parts(d, group, counts, lens):
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + group)
    pg, K, V = _pool(lens, 16, d, BF, gen)
    T, starts = sum(counts), [sum(counts[:b]) for b in range(len(counts) + 1)]
    q = torch.randn((T, group, d), generator=gen).to(BF)
    assert max(counts) * group <= 32   # (calls that name their longest sequence)
    o, lse = (x.cpu() for x in G.chunk_attention(q.cuda(), pg, _i32(starts), heads=1, longest=max(counts),
                                                 return_lse=True))
    for b, c in enumerate(counts):
        at = slice(starts[b], starts[b + 1])
        for g in range(group if c else 0):
            _close("seq %d head %d" % (b, g), o[at, g], lse[at, g], q[at, g], K[b], V[b], sink_seen(lens[b], c, 0, 0))


@pytest.mark.parametrize("dtype,d,group,counts,lens", [
    (BF, 128, 4, [1, 2], [300, 40]), (BF, 64, 4, [1, 1], [900, 20000]), (F32, 128, 4, [2, 20], [500, 90]),
    (F32, 64, 1, [1, 1], [100, 17]), (BF, 128, 4, [100, 1], [700, 50]), (BF, 64, 5, [40, 60], [1500, 400])])
def test_large_values_under_growing_logits(dtype, d, group, counts, lens):
    # logits that rise by 39 (log2) along the keys under values of 1e36: no weight against an early
    # reference may carry finite values past a float's range
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + group)
    pg, K, V = _pool(lens, 64, d, dtype, gen)
    T, starts = sum(counts), [sum(counts[:b]) for b in range(len(counts) + 1)]
    q = torch.randn((T, group, d), generator=gen)
    for u, n in enumerate(lens):
        K[u], V[u] = K[u].float(), V[u].float()
        _ramp(q, K[u], V[u], -19.5, 19.5)
        K[u], V[u] = K[u].to(dtype), V[u].to(dtype)
        slot = torch.arange(n, device="cuda")
        pg.k[pg.table[u, slot // 64].long(), slot % 64] = K[u].cuda()
        pg.v[pg.table[u, slot // 64].long(), slot % 64] = V[u].cuda()
    q = q.to(dtype)
    o, lse = (x.cpu() for x in G.chunk_attention(q.cuda(), pg, _i32(starts), heads=1, return_lse=True))
    assert torch.isfinite(o).all()
    for b, c in enumerate(counts):
        at = slice(starts[b], starts[b + 1])
        for g in range(group):
            check("seq %d head %d" % (b, g), o[at, g], lse[at, g], q[at, g], K[b], V[b], sink_seen(lens[b], c, 0, 0))


def test_infinities_that_every_row_sees_stay_infinities():
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(21)
    for dtype, c in ((BF, 1), (BF, 30), (F32, 1), (F32, 30)):
        pg, K, V = _pool([700], 64, 128, dtype, gen)
        V[0][70, 7], V[0][70, 9] = torch.inf, -torch.inf
        pg.v[int(pg.table[0, 1]), 6] = V[0][70].cuda()
        q = torch.randn((c, 4, 128), generator=gen).to(dtype)
        o = G.chunk_attention(q.cuda(), pg, _i32([0, c]), heads=1).cpu()
        assert (o[..., 7] == torch.inf).all() and (o[..., 9] == -torch.inf).all()
        assert torch.isfinite(o[..., [x for x in range(128) if x not in (7, 9)]]).all()


def test_results_do_not_depend_on_the_workspace_or_the_run():
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(7)
    lens, counts = [5000, 40, 900, 3000], [1, 30, 200, 2]
    pg, _, _ = _pool(lens, 64, 128, BF, gen)
    q = torch.randn((sum(counts), 4, 128), generator=gen).to(BF).cuda()
    starts = _i32([0, 1, 31, 231, 233])
    ws = torch.empty(G.chunk_attention_workspace_bytes(pg, 4, 1, 233, 4), dtype=torch.uint8, device="cuda")
    first = None
    for fill in (0, 255, 127):
        ws.fill_(fill)
        o, lse = G.chunk_attention(q, pg, starts, heads=1, return_lse=True, workspace=ws)
        if first is None:
            first = o, lse
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


def test_captured_calls_and_another_stream():
    # lengths and starts change between the replays; two graphs over one workspace
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(11)
    B, H, group, d, T = 4, 2, 4, 64, 80
    pg, _, _ = _pool([700] * (B * H), 16, d, BF, gen)
    pg.k.nan_to_num_(0.0)
    pg.v.nan_to_num_(0.0)
    q = torch.randn((T, H * group, d), generator=gen).to(BF).cuda()
    starts = _i32([0, 1, 2, 60, 61])
    ws = torch.empty(G.chunk_attention_workspace_bytes(pg, B, H, T, group), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(q), torch.zeros_like(q)]
    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            G.chunk_attention(q, pg, starts, heads=H, out=out, workspace=ws)
        graphs.append(g)
    for turn in range(4):
        starts.copy_(_i32([0, 5 * turn, 5 * turn, 50 + turn, T]))
        pg.lens[:B * H] = 700 - 130 * turn
        want = G.chunk_attention(q, pg, starts, heads=H)
        for g, out in zip(graphs, outs):
            out.zero_()
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = G.chunk_attention(q, pg, starts, heads=H, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o, want)


def test_agrees_with_the_calls_beside_it():
    # a chain of drafted tokens, and a prompt over contiguous keys: the same rows, other kernels or
    # other cuts; each within its bounds of the formula, so within twice those of each other
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(13)
    d, n, c, group = 128, 500, 12, 4
    pg, K, V = _pool([n, n], 64, d, BF, gen)
    q = torch.randn((2, c, group, d), generator=gen).to(BF).cuda()
    o, lse = G.chunk_attention(q.view(2 * c, group, d), pg, _i32([0, c, 2 * c]), heads=1, return_lse=True)
    qt = q.transpose(1, 2).contiguous()
    to, tl = G.tree_attention(qt, pg, units=_i32([0, 1]), return_lse=True)
    so, sl = G.sink_attention(qt, torch.stack(K).cuda(), torch.stack(V).cuda(), 0, return_lse=True)
    for x, l in ((to, tl), (so, sl)):
        for e in range(2):
            for g in range(group):
                check("beside", x[e, g].cpu(), l[e, g].cpu(), qt[e, g].cpu(), K[e], V[e], sink_seen(n, c, 0, 0))
    for e in range(2):
        for g in range(group):
            at = slice(e * c, e * c + c)
            check("chunk", o[at, g].cpu(), lse[at, g].cpu(), qt[e, g].cpu(), K[e], V[e], sink_seen(n, c, 0, 0))


def test_units_of_a_layer():
    # a layer's columns of a model's units
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(17)
    B, L, H, group, d = 3, 2, 2, 2, 64
    lens = [20 + 9 * u for u in range(B * L * H)]
    pg, K, V = _pool(lens, 16, d, BF, gen)
    every = torch.arange(B * L * H, dtype=torch.int32, device="cuda").view(B, L, H)
    counts = [1, 12, 3]
    q = torch.randn((16, H * group, d), generator=gen).to(BF)
    for layer in range(L):
        o, lse = (x.cpu() for x in G.chunk_attention(q.cuda(), pg, _i32([0, 1, 13, 16]), units=every[:, layer],
                                                     return_lse=True))
        at = 0
        for b, c in enumerate(counts):
            for h in range(H):
                u = (b * L + layer) * H + h
                for x in range(h * group, (h + 1) * group):
                    check("layer %d" % layer, o[at:at + c, x], lse[at:at + c, x], q[at:at + c, x], K[u], V[u],
                          sink_seen(lens[u], c, 0, 0))
            at += c


def test_binding_checks():
    import paper_2605_31105_amd as G
    pg = G.new_pages(4, 4, 16, 16, 64)
    q, starts = torch.zeros((3, 4, 64), dtype=BF, device="cuda"), _i32([0, 1, 3])
    for call in (lambda: G.chunk_attention(q, pg, starts), lambda: G.chunk_attention(q.float(), pg, starts, heads=2),
                 lambda: G.chunk_attention(q, pg, starts, heads=3), lambda: G.chunk_attention(q[0], pg, starts, heads=2),
                 lambda: G.chunk_attention(q, pg, starts.long(), heads=2), lambda: G.chunk_attention(q.cpu(), pg, starts, heads=2),
                 lambda: G.chunk_attention(q[..., :32].contiguous(), pg, starts, heads=2),
                 lambda: G.chunk_attention(q.transpose(0, 1), pg, starts, heads=1), lambda: G.chunk_attention(q, pg, starts[:0], heads=2),
                 lambda: G.chunk_attention(q, pg, starts, heads=2, out=q[:2]), lambda: G.chunk_attention(q, pg, starts, units=_i32([[0, 1]])),
                 lambda: G.chunk_attention(q, pg, starts, heads=2, window=1 << 31)):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(window=-1), dict(n_sink=-1), dict(longest=0)):
        with pytest.raises(G.GrkvError) as e:
            G.chunk_attention(q, pg, starts, heads=2, **kw)
        assert e.value.status == G.GRKV_ERR_INVALID
    assert G.chunk_attention(q[:0], pg, _i32([0, 0]), heads=2).shape == (0, 4, 64)
    assert G.chunk_attention_workspace_bytes(pg, 2, 2, 3, 2, longest=0) == 0


def _two_parts(c, group):
    """Whether the weights of each (token, head of the group) of a sequence of c new tokens are held to two
    parts: those of its last 64 rows or fewer past a multiple of 128, rows being token by token."""
    r = torch.arange(c * group).view(c, group)
    return (r >= c * group // 128 * 128) & (c * group % 128 <= 64)


@pytest.mark.parametrize("d,group,counts,lens", [
    (128, 4, [16, 300, 9, 1], [300, 520, 40, 2000]), (64, 3, [21, 5, 70, 0], [129, 33, 300, 4]),
    (128, 7, [9] * 40, [30 + 31 * b for b in range(40)]), (64, 16, [4, 2, 3], [9000, 20, 700]),
    (128, 1, [64, 33, 190, 65], [64, 1000, 250, 400]), (64, 5, [12] * 70 + [200], [40 + 17 * b for b in range(70)] + [900])])
def test_weights_of_up_to_64_rows_are_held_to_two_parts(d, group, counts, lens):
    # whatever the other sequences are, and whether the call names its longest or not
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + group)
    pg, K, V = _pool(lens, 16, d, BF, gen)
    T, starts = sum(counts), [sum(counts[:b]) for b in range(len(counts) + 1)]
    q = torch.randn((T, group, d), generator=gen).to(BF)
    for longest in (None, max(counts)):
        o, lse = (x.cpu() for x in G.chunk_attention(q.cuda(), pg, _i32(starts), heads=1, longest=longest, return_lse=True))
        done = 0
        for b, c in enumerate(counts):
            two = _two_parts(c, group)
            for g in range(group):
                at = two[:, g].nonzero().flatten() if c else torch.zeros(0, dtype=torch.long)
                if at.numel() == 0:
                    continue
                done += at.numel()
                x = starts[b] + at
                _close("seq %d head %d" % (b, g), o[x, g], lse[x, g], q[x, g], K[b], V[b], sink_seen(lens[b], c, 0, 0)[at])
        assert done >= 4 * group


@pytest.mark.parametrize("d,window,n_sink", [(128, 50, 5), (64, 37, 70)])
def test_up_to_64_rows_with_windows(d, window, n_sink):
    counts, before = [16, 9, 40, 11], [900, 100, 3000, 0]
    lens = [[b + 5 * h + c for h in range(2)] for b, c in zip(before, counts)]
    _run("64", lens, counts, 2, 4, 16, d, BF, window, n_sink, pad=2)


@pytest.mark.parametrize("group,counts", [(8, [6]), (16, [4, 1]), (5, [11, 20])])
def test_what_up_to_64_rows_do_not_see_never_reaches_them(group, counts):
    test_what_a_query_does_not_see_never_reaches_it(BF, group, counts)


@pytest.mark.parametrize("d,group,counts,lens", [(128, 5, [12, 40], [700, 900]), (64, 16, [4, 3], [20000, 300]), (128, 1, [60], [1500])])
def test_large_values_under_growing_logits_of_up_to_64_rows(d, group, counts, lens):
    test_large_values_under_growing_logits(BF, d, group, counts, lens)


def test_infinities_that_up_to_64_rows_see_stay_infinities():
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(22)
    for d, n in ((128, 700), (64, 9000)):
        pg, K, V = _pool([n], 64, d, BF, gen)
        V[0][70, 7], V[0][70, 9] = torch.inf, -torch.inf
        pg.v[int(pg.table[0, 1]), 6] = V[0][70].cuda()
        q = torch.randn((13, 4, d), generator=gen).to(BF)
        o = G.chunk_attention(q.cuda(), pg, _i32([0, 13]), heads=1).cpu()
        assert (o[..., 7] == torch.inf).all() and (o[..., 9] == -torch.inf).all()
        assert torch.isfinite(o[..., [x for x in range(d) if x not in (7, 9)]]).all()


@pytest.mark.parametrize("dtype,d,group,counts,before,window,n_sink", [
    # up to 16 rows a unit: few units, whose blocks join their pieces, and many, cut into equal parts
    (BF, 128, 4, [1, 3], [5000, 2070], 1000, 37), (BF, 64, 5, [2, 1, 0], [3001, 40, 900], 333, 5),
    (BF, 128, 4, [1] * 50, [19 + 61 * b for b in range(50)], 77, 13), (BF, 64, 16, [1] * 70, [5 + 43 * b for b in range(70)], 100, 70),
    # 17 to 32 rows: pieces of a job a block, and equal parts
    (BF, 128, 4, [5, 8, 1], [4000, 333, 0], 1000, 37), (BF, 64, 3, [10, 6], [2100, 50], 333, 70),
    (BF, 128, 7, [4, 3] * 25, [20 + 61 * b for b in range(50)], 77, 13), (BF, 64, 4, [8, 1] * 35, [5 + 43 * b for b in range(70)], 100, 5),
    # float32: 16 rows a unit, and tiles of 32
    (F32, 128, 4, [1, 3], [3000, 70], 333, 37), (F32, 64, 4, [8, 1] * 20, [5 + 43 * b for b in range(40)], 77, 13),
    (F32, 128, 3, [10, 20], [2100, 50], 333, 5),
    # windows of a slot or two, and shorter than the new tokens
    (BF, 128, 4, [4, 1], [500, 70], 1, 0), (BF, 64, 2, [15, 9], [300, 2], 2, 33), (BF, 128, 4, [7, 2], [500, 70], 3, 1)])
def test_windows_of_calls_that_name_their_longest(dtype, d, group, counts, before, window, n_sink):
    lens = [[b + 3 * h + c for h in range(2)] for b, c in zip(before, counts)]
    few = len(counts) < 10
    _run("named", lens, counts, 2, group, 16, d, dtype, window, n_sink, pad=1, longest=max(counts), heads=None if few else [1])


@pytest.mark.parametrize("d,dtype,sequences,longest", [(128, BF, 5, None), (64, BF, 90, None), (128, BF, 90, 4), (64, BF, 5, 4),
                                                       (128, BF, 90, 8), (64, F32, 90, None), (128, F32, 5, 4)])
def test_starts_that_fall_or_pass_the_rows_stay_inside_them(d, dtype, sequences, longest):
    # q lies between rows of NaN, o, lse and the workspace between marks: nothing beside them is read
    # or written
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + sequences)
    group, T, edge = 4, 120, 40
    pg, _, _ = _pool([10 + (37 * b) % 500 for b in range(sequences)], 16, d, dtype, gen)
    pg.k.nan_to_num_(0.0)
    pg.v.nan_to_num_(0.0)
    q = torch.full((T + 2 * edge, group, d), math.nan, dtype=dtype, device="cuda")
    q[edge:-edge] = torch.randn((T, group, d), generator=gen).to(dtype).cuda()
    o, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 6.0, device="cuda")
    need = G.chunk_attention_workspace_bytes(pg, sequences, 1, T, group, longest)
    ws = torch.full((need + 2 * 4096,), 165, dtype=torch.uint8, device="cuda")
    at = slice(edge, T + edge)
    some = torch.randint(-T, 2 * T, (6, sequences + 1), generator=gen).tolist()
    far = [[(1 << 30) * (b % 3 - 1) for b in range(sequences + 1)], [2 ** 31 - 1 - b for b in range(sequences + 1)],
           [T - b for b in range(sequences + 1)], [-(2 ** 31)] + [T] * sequences, [0] + [2 ** 31 - 1] * sequences]
    for starts in some + far:
        o.fill_(5.0)
        lse.fill_(6.0)
        G.chunk_attention(q[at], pg, _i32(starts), heads=1, longest=longest, out=o[at], lse=lse[at],
                          workspace=ws[4096:4096 + need])
        torch.cuda.synchronize()
        for x, mark in ((o, 5.0), (lse, 6.0)):
            assert (x[:edge] == mark).all() and (x[-edge:] == mark).all()
        assert (ws[:4096] == 165).all() and (ws[4096 + need:] == 165).all()
        assert torch.isfinite(o).all() and not torch.isnan(lse).any()
