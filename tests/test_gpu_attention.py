"""Attention over pages (tree_attention) and with a window and sinks over contiguous keys
(sink_attention) against float64 rows, within the bounds of tests/attention_ref.py."""
import math

import pytest

from tests.attention_ref import check, rows, sink_seen, tree_seen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pool(lens, ps, d, dtype, gen, scale=1.0):
    """A pool of NaN whose units hold random rows, its pages scattered; rows on the host."""
    import paper_2605_31105_amd as G
    held = [-(-n // ps) for n in lens]
    pages = 2 * sum(held) + 3
    pg = G.new_pages(len(lens) + 1, max(held + [1]) + 1, pages, ps, d, dtype)
    pg.k.fill_(math.nan)
    pg.v.fill_(math.nan)
    ids = torch.randperm(pages, generator=gen)
    K, V, at = [], [], 0
    for u, n in enumerate(lens):
        K.append((torch.randn((n, d), generator=gen) * scale).to(dtype))
        V.append(torch.randn((n, d), generator=gen).to(dtype))
        for j in range(held[u]):
            p = int(ids[at])
            at += 1
            rows_ = slice(j * ps, min(n, (j + 1) * ps))
            m = rows_.stop - rows_.start
            pg.k[p, :m] = K[u][rows_].cuda()
            pg.v[p, :m] = V[u][rows_].cuda()
            pg.table[u, j] = p
        pg.lens[u] = n
    return pg, K, V


def _parents(kind, trees, t, gen):
    if kind == "chain":
        return None, [list(range(-1, t - 1))] * trees
    if kind == "flat":
        p = [[-1] * t] * trees
    elif kind == "bad":    # not earlier tokens: they count as none
        p = [[(-5, i, 100, i - 1)[i % 4] for i in range(t)] for _ in range(trees)]
    else:
        p = [[int(torch.randint(-1, i, (1,), generator=gen)) if i else -1 for i in range(t)]
             for _ in range(trees)]
    return _i32(p), p


TREE_CASES = [
    # dtype, d, page, group, tokens, lens, parents, window, sinks
    (BF, 128, 64, 4, 1, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 1000, 5000], "chain", 0, 0),
    (BF, 64, 16, 1, 5, [0, 3, 5, 6, 20, 33, 200, 4097], "tree", 0, 0),
    (BF, 128, 32, 5, 33, [33, 34, 100, 2049], "tree", 0, 0),
    (BF, 128, 256, 8, 64, [64, 70, 700], "tree", 0, 0),
    (BF, 64, 128, 3, 9, [9, 400, 1300], "bad", 0, 0),
    (BF, 128, 16, 2, 4, [4, 50, 900, 3000], "flat", 37, 4),
    (BF, 64, 64, 7, 2, [2, 640, 641, 2100], "chain", 500, 70),
    (BF, 128, 64, 4, 33, [40, 77, 1000], "tree", 1, 0),
    (BF, 128, 64, 4, 12, [12, 13, 400], "chain", 5, 14),
    (BF, 128, 1024, 1, 1, [1, 1023, 1024, 1025, 9000], "chain", 100, 0),
    (F32, 128, 32, 3, 7, [3, 7, 8, 100, 1500], "tree", 50, 4),
    (F32, 64, 256, 8, 64, [64, 65, 300, 1025], "chain", 10, 2),
    (F32, 64, 16, 1, 1, [0, 1, 15, 16, 17, 500], "chain", 0, 0),
    (F32, 128, 64, 6, 6, [6, 2000], "tree", 0, 0),
]


@pytest.mark.parametrize("case", TREE_CASES, ids=lambda c: "%s-d%d-p%d-g%d-t%d-%s-w%d" % (
    "bf16" if c[0] == BF else "f32", c[1], c[2], c[3], c[4], c[6], c[7]))
def test_tree_attention(case):
    import paper_2605_31105_amd as G
    dtype, d, ps, group, t, lens, kind, window, n_sink = case
    gen = torch.Generator().manual_seed(d + ps + t)
    pg, K, V = _pool(lens, ps, d, dtype, gen)
    E = len(lens)
    trees = 2 if E % 2 == 0 else 1
    parents, plist = _parents(kind, trees, t, gen)
    q = torch.randn((E, group, t, d), generator=gen).to(dtype)
    units = torch.randperm(E, generator=gen).tolist()
    o, lse = G.tree_attention(q.cuda(), pg, parents, units=_i32(units), window=window, n_sink=n_sink,
                              return_lse=True)
    torch.cuda.synchronize()
    for e, u in enumerate(units):
        seen = tree_seen(lens[u], t, plist[e // (E // trees)], window, n_sink)
        for g in range(group):
            check("len %d head %d" % (lens[u], g), o[e, g].cpu(), lse[e, g].cpu(), q[e, g], K[u], V[u], seen)


def test_tree_attention_padded_batch_and_bad_units():
    # ragged drafted tokens: rows behind counts stay as they were; a unit twice; no such unit
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(9)
    lens = [100, 37, 3, 64]
    pg, K, V = _pool(lens, 16, 64, BF, gen)
    t, group = 6, 3
    units, counts = [0, 1, 1, 3, 2, -1, 99, 4], [6, 0, 2, 9, 5, 2, 3, 1]
    parents, plist = _parents("tree", 1, t, gen)
    q = torch.randn((8, group, t, 64), generator=gen).to(BF)
    o = torch.full(q.shape, 5.0, dtype=BF, device="cuda")
    lse = torch.full(q.shape[:3], 6.0, device="cuda")
    G.tree_attention(q.cuda(), pg, parents, units=_i32(units), counts=_i32(counts), out=o, lse=lse)
    torch.cuda.synchronize()
    o, lse = o.cpu(), lse.cpu()
    empty = torch.zeros((0, 64), dtype=BF)
    for e, (u, c) in enumerate(zip(units, counts)):
        c = min(c, t)
        assert (o[e, :, c:] == 5).all() and (lse[e, :, c:] == 6).all()
        n, Ku, Vu = (lens[u], K[u], V[u]) if 0 <= u < 4 else (0, empty, empty)
        for g in range(group):
            check("entry %d" % e, o[e, g, :c], lse[e, g, :c], q[e, g, :c], Ku, Vu,
                  tree_seen(n, c, plist[0], 0, 0))


@pytest.mark.parametrize("dtype,group,tokens", [(BF, 2, 6), (F32, 2, 6), (BF, 16, 6), (BF, 48, 6)])
def test_what_a_query_does_not_see_never_reaches_it(dtype, group, tokens):
    # NaN and infinities in the keys and values of a sibling: the rows that do not see it are
    # within their bounds of the finite cache's, those that do are not finite.  (Such a tile is
    # summed key by key, with other references than the products', so a weight may be rounded
    # the other way: the bounds of attention_ref hold for both, a comparison of the two in
    # steps of o does not.)
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(3)
    plist = [[-1, 0, 0, 1, 2, 4]]
    parents = _i32(plist)
    pg, K, V = _pool([70], 16, 64, dtype, gen)
    q = torch.randn((1, group, tokens, 64), generator=gen).to(dtype)
    seen = tree_seen(70, 6, plist[0], 0, 0)
    for where, value in ((2, math.nan), (2, math.inf), (5, -math.inf), (3, math.nan)):
        slot = 64 + where
        page, row = int(pg.table[0, slot // 16]), slot % 16
        see = seen[:, slot]
        for t in (pg.k, pg.v):
            keep = t[page, row].clone()
            t[page, row] = value
            o, lse = (x[0].cpu() for x in G.tree_attention(q.cuda(), pg, parents, units=_i32([0]), return_lse=True))
            t[page, row] = keep
            for g in range(group):
                check("slot %d %s head %d" % (slot, value, g), o[g, ~see], lse[g, ~see], q[0, g, ~see],
                      K[0], V[0], seen[~see])
            if t is pg.v or math.isnan(value):
                assert not torch.isfinite(o[:, see]).all()


def test_large_logits_move_the_reference():
    # logits that grow along the cache by thousands, and a key far above all others
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(5)
    for dtype in (BF, F32):
        pg, K, V = _pool([2000], 64, 128, dtype, gen)
        q = torch.randn((1, 4, 2, 128), generator=gen)
        q[0, 0, 0] = 0
        q[0, 0, 0, 0] = 64.0
        ramp = torch.linspace(-400, 400, 2000)
        K[0][:, 0] = ramp.to(dtype)
        K[0][777] = (K[0][777].float() * 300).to(dtype)
        q = q.to(dtype)
        pages = pg.table[0, torch.arange(2000, device="cuda") // 64].long()
        pg.k[pages, torch.arange(2000, device="cuda") % 64] = K[0].cuda()
        o, lse = G.tree_attention(q.cuda(), pg, units=_i32([0]), return_lse=True)
        torch.cuda.synchronize()
        seen = tree_seen(2000, 2, [-1, 0], 0, 0)
        for g in range(4):
            check("head %d" % g, o[0, g].cpu(), lse[0, g].cpu(), q[0, g], K[0], V[0], seen)


SINK_CASES = [
    # dtype, d, U, G, n, nq, window, sinks
    (BF, 128, 1, 1, 1, 1, 0, 0), (BF, 64, 2, 3, 17, 17, 4, 1), (BF, 128, 2, 4, 300, 300, 64, 4),
    (BF, 128, 1, 4, 1000, 1000, 0, 0), (BF, 128, 2, 5, 700, 37, 100, 9), (BF, 64, 3, 8, 2500, 1, 500, 4),
    (BF, 128, 1, 2, 513, 513, 1, 0), (BF, 64, 1, 1, 400, 399, 37, 50), (BF, 128, 1, 7, 200, 130, 1000, 4),
    (BF, 128, 1, 1, 1500, 1500, 256, 300), (BF, 64, 2, 16, 130, 70, 33, 2), (BF, 128, 3, 4, 4100, 2, 0, 0),
    (F32, 128, 1, 3, 259, 259, 50, 4), (F32, 64, 2, 5, 700, 101, 77, 9), (F32, 128, 2, 4, 1200, 1, 100, 0),
    (F32, 64, 1, 1, 600, 600, 0, 0),
]


@pytest.mark.parametrize("case", SINK_CASES, ids=lambda c: "%s-d%d-u%d-g%d-n%d-q%d-w%d-s%d" % (
    ("bf16" if c[0] == BF else "f32",) + c[1:]))
def test_sink_attention(case):
    import paper_2605_31105_amd as G
    dtype, d, U, group, n, nq, window, n_sink = case
    gen = torch.Generator().manual_seed(n + nq + d)
    q = torch.randn((U, group, nq, d), generator=gen).to(dtype)
    K, V = (torch.randn((U, n, d), generator=gen).to(dtype) for _ in range(2))
    o, lse = G.sink_attention(q.cuda(), K.cuda(), V.cuda(), window, n_sink, return_lse=True)
    torch.cuda.synchronize()
    seen = sink_seen(n, nq, window, n_sink)
    for u in range(U):
        for g in range(group):
            check("unit %d head %d" % (u, g), o[u, g].cpu(), lse[u, g].cpu(), q[u, g], K[u], V[u], seen)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_later_keys_that_are_not_finite_do_not_reach_earlier_queries(dtype):
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(8)
    n = 200
    q = torch.randn((1, 2, n, 64), generator=gen).to(dtype)
    K, V = (torch.randn((1, n, 64), generator=gen).to(dtype) for _ in range(2))
    bad = V.clone()
    bad[0, 101] = math.nan
    bad[0, 103, 5] = math.inf
    got, lse = (x.cpu() for x in G.sink_attention(q.cuda(), K.cuda(), bad.cuda(), 50, 3, return_lse=True))
    clean = torch.ones(n, dtype=torch.bool)
    clean[101:153] = False
    seen = sink_seen(n, n, 50, 3)[clean]
    for g in range(2):
        check("head %d" % g, got[0, g, clean], lse[0, g, clean], q[0, g, clean], K[0], V[0], seen)
    assert torch.isnan(got[0, :, 101:151]).all()
    assert torch.isinf(got[0, :, 151:153, 5]).all()


def test_windows_and_sinks_of_every_size():
    # up to the largest int, which is no window: the rows of the smallest that holds all
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(12)
    q = torch.randn((1, 2, 100, 64), generator=gen).to(BF).cuda()
    K, V = (torch.randn((1, 100, 64), generator=gen).to(BF).cuda() for _ in range(2))
    want = G.sink_attention(q, K, V, 0)
    big = (1 << 31) - 1
    for window, n_sink in ((100, 0), (101, 4), (1 << 30, 0), (big, big), (1, big), (3, 100), (99, 1)):
        if window >= 100:
            assert torch.equal(G.sink_attention(q, K, V, window, n_sink), want)
        check("window %d sinks %d" % (window, n_sink), *(x[0, 1].cpu() for x in G.sink_attention(
            q, K, V, window, n_sink, return_lse=True)), q[0, 1].cpu(), K[0].cpu(), V[0].cpu(),
            sink_seen(100, 100, window, n_sink))
    pg, Kt, Vt = _pool([90, 2], 16, 64, BF, gen)
    qt = torch.randn((2, 2, 5, 64), generator=gen).to(BF)
    for window, n_sink in ((big, big), (1 << 30, 3), (1, big), (112, 0), (4, 88)):
        o, lse = G.tree_attention(qt.cuda(), pg, units=_i32([0, 1]), window=window, n_sink=n_sink, return_lse=True)
        for u, n in ((0, 90), (1, 2)):
            check("unit %d window %d" % (u, window), o[u, 0].cpu(), lse[u, 0].cpu(), qt[u, 0], Kt[u], Vt[u],
                  tree_seen(n, 5, [-1, 0, 1, 2, 3], window, n_sink))


def test_window_calls_agree_with_each_other():
    # the last queries of a prompt, a chunk of it and single tokens give the prompt's rows
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(2)
    q = torch.randn((2, 4, 777, 128), generator=gen).cuda()
    K, V = (torch.randn((2, 777, 128), generator=gen).cuda() for _ in range(2))
    whole = G.sink_attention(q, K, V, 100, 4)
    part = G.sink_attention(q[:, :, 700:].contiguous(), K, V, 100, 4)
    assert (whole[:, :, 700:] - part).abs().max() < 1e-5
    for p in (0, 3, 4, 99, 104, 500):
        one = G.sink_attention(q[:, :, p:p + 1].contiguous(), K[:, :p + 1].contiguous(),
                               V[:, :p + 1].contiguous(), 100, 4)
        assert (whole[:, :, p:p + 1] - one).abs().max() < 1e-5


@pytest.mark.parametrize("units,group,tokens", [(8, 4, 1), (300, 2, 1), (700, 1, 3), (4, 8, 64)])
def test_long_units_with_and_without_splits(units, group, tokens):
    # splits are a matter of the call's size: against torch in float64 on the GPU
    import paper_2605_31105_amd as G
    g = torch.Generator(device="cuda").manual_seed(units)
    n, ps, d = 1500 if units > 100 else 9000, 64, 128
    held = -(-n // ps)
    pg = G.new_pages(units, held, units * held, ps, d)
    k = torch.randn((units, n, d), device="cuda", generator=g).to(BF)
    v = torch.randn((units, n, d), device="cuda", generator=g).to(BF)
    assert not G.pages_append(pg, k, v).any().item()
    q = torch.randn((units, group, tokens, d), device="cuda", generator=g).to(BF)
    o, lse = G.tree_attention(q, pg, return_lse=True)
    again, _ = G.tree_attention(q, pg, return_lse=True)
    assert torch.equal(o, again)
    for u in (0, units // 2, units - 1):
        seen = tree_seen(n, tokens, list(range(-1, tokens - 1)), 0, 0)
        for h in range(0, group, 3):
            check("unit %d" % u, o[u, h].cpu(), lse[u, h].cpu(), q[u, h].cpu(), k[u].cpu(), v[u].cpu(), seen)


@pytest.mark.parametrize("group,tokens,n", [(4, 1, 2000), (2, 9, 1500), (4, 40, 3000), (1, 1, 40000)])
def test_splits_do_not_depend_on_what_the_workspace_held(group, tokens, n):
    # splits that blocks join themselves, and those combined by a second launch: with a
    # workspace of ones, of zeros and of the last call's, the same rows bit for bit
    import paper_2605_31105_amd as G
    gen = torch.Generator(device="cuda").manual_seed(n)
    pg = G.new_pages(3, -(-n // 64), 3 * -(-n // 64), 64, 128)
    k, v = (torch.randn((3, n, 128), device="cuda", generator=gen).to(BF) for _ in range(2))
    assert not G.pages_append(pg, k, v).any().item()
    q = torch.randn((3, group, tokens, 128), device="cuda", generator=gen).to(BF)
    need = G.tree_attention_workspace_bytes(pg, 3, group, tokens)
    assert need > 256
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    want, lse = G.tree_attention(q, pg, workspace=ws, return_lse=True)
    for fill in (None, 0, 1, None, None):
        if fill is not None:
            ws.fill_(fill)
        got, l2 = G.tree_attention(q, pg, workspace=ws, return_lse=True)
        assert torch.equal(got, want) and torch.equal(l2, lse)
    seen = tree_seen(n, tokens, list(range(-1, tokens - 1)), 0, 0)
    check("unit 2", want[2, 0].cpu(), lse[2, 0].cpu(), q[2, 0].cpu(), k[2].cpu(), v[2].cpu(), seen)


def test_captured_calls_and_another_stream():
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(4)
    pg, K, V = _pool([900, 50], 64, 128, BF, gen)
    q = torch.randn((2, 4, 3, 128), generator=gen).to(BF).cuda()
    Kc, Vc = (torch.randn((2, 300, 128), generator=gen).to(BF).cuda() for _ in range(2))
    units = _i32([0, 1])
    want = G.tree_attention(q, pg, units=units), G.sink_attention(q, Kc, Vc, 64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = G.tree_attention(q, pg, units=units, stream=side), G.sink_attention(q, Kc, Vc, 64, stream=side)
    handle = G.tree_attention(q, pg, units=units, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and torch.equal(handle, want[0])
    outs = torch.empty_like(q), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.tree_attention(q, pg, units=units, out=outs[0])
        G.sink_attention(q, Kc, Vc, 64, out=outs[1])
    for _ in range(3):
        outs[0].zero_()
        outs[1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
        assert torch.equal(G.tree_attention(q, pg, units=units), want[0])
    # a length that grew since the capture is the one read
    pg.lens[1] = 49
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], G.tree_attention(q, pg, units=units))


def test_compress_store_attend_and_draft():
    """The path as it is used: a cache is compressed, stored, attended to by its window (which
    gives the discrepancy that the compression reported), extended by drafted tokens, and taken
    down to the accepted ones."""
    import paper_2605_31105_amd as G
    import workloads as W
    from tests.parity import to_device
    cfg = W.config(2, layers=1, kv_heads=2, n=2048, budget=256)
    q, K, V = (to_device(a, cfg.dtype) for a in W.make_batch(cfg))
    U, c, d, w = cfg.units, cfg.budget, cfg.head_dim, cfg.window
    res = G.compress(q, K, V, w, c, cfg.pool_kernel, cfg.lam)
    pg = G.new_pages(U + 2, 12, 60, 32, d, F32)
    assert not G.pages_append(pg, res.k_out, res.v_out).any().item()
    # the window's queries are the last w slots as a chain: o = X V*
    o = G.tree_attention(q.float(), pg, units=_i32([0, 1]))
    Y = G.intermediates(res)["y"].view(U, cfg.group, w, d)
    D = ((Y - o).double().square().sum((1, 2, 3)) / Y.double().square().sum((1, 2, 3))).cpu()
    want = res.stats[:, 2].double().cpu()
    print("D", D.tolist(), "reported", want.tolist(), flush=True)
    assert ((D - want).abs() <= 2e-3 * want + 1e-9).all()
    # ragged results go in packed, by their budgets and offsets
    idx, k_out, v_out, _, offs = G.compress_ragged(q, K, V, w, [200, 77], cfg.pool_kernel, cfg.lam)
    st = G.pages_append(pg, k_out, v_out, units=_i32([2, 3]), counts=_i32([200, 77]),
                        starts=torch.from_numpy(offs).cuda(), rows=200)
    assert not st.any().item() and pg.lens.tolist() == [256, 256, 200, 77]
    o2 = G.tree_attention(q.float(), pg, units=_i32([2, 3]))
    for u, (n, at) in enumerate(((200, 0), (77, 200))):
        seen = tree_seen(n, w, list(range(-1, w - 1)), 0, 0)
        for g in range(cfg.group):
            want = rows(q[u, g].float().cpu(), k_out[at:at + n].float().cpu(), v_out[at:at + n].cpu(),
                        seen, False)
            assert ((o2[u, g].cpu().double() - want[0]).abs() <= want[2]).all()
    # four drafted tokens, a tree; tokens 0, 2 and 3 are accepted
    gen = torch.Generator().manual_seed(1)
    kd, vd, qd = (torch.randn(s, generator=gen).cuda() for s in ((2, 4, d), (2, 4, d), (2, 4, 4, d)))
    tree = _i32([[-1, 0, 0, 2]])
    u01 = _i32([0, 1])
    G.pages_append(pg, kd, vd, units=u01)
    tree_o = G.tree_attention(qd, pg, tree, units=u01)
    st = G.pages_compact(pg, _i32([[256, 258, 259]] * 2), units=u01, keep=_i32([256, 256]))
    assert not st.any().item() and pg.lens[:2].tolist() == [259, 259]
    chain_o = G.tree_attention(qd[:, :, [0, 2, 3]].contiguous(), pg, units=u01)
    assert (chain_o - tree_o[:, :, [0, 2, 3]]).abs().max() < 1e-5
    G.pages_free(pg)
    assert pg.free.tolist() == [-1, (1 << 28) - 1]


def test_binding_checks():
    import paper_2605_31105_amd as G
    pg = G.new_pages(4, 4, 8, 16, 64)
    q = torch.zeros(4, 2, 3, 64, dtype=BF, device="cuda")
    K = torch.zeros(4, 5, 64, dtype=BF, device="cuda")
    for call in (lambda: G.tree_attention(q.float(), pg), lambda: G.tree_attention(q.cpu(), pg),
                 lambda: G.tree_attention(q.transpose(1, 2), pg), lambda: G.tree_attention(q[0], pg),
                 lambda: G.tree_attention(q[..., :32].contiguous(), pg),
                 lambda: G.tree_attention(q, pg, _i32([-1, 0, 1])),
                 lambda: G.tree_attention(q, pg, _i32([[-1, 0]])),
                 lambda: G.tree_attention(q, pg, counts=_i32([1])),
                 lambda: G.tree_attention(q, pg, units=torch.zeros(4, device="cuda")),
                 lambda: G.tree_attention(q, pg, out=torch.zeros_like(K)),
                 lambda: G.tree_attention(q, pg, lse=torch.zeros(4, device="cuda")),
                 lambda: G.sink_attention(q, K, K.float(), 4), lambda: G.sink_attention(q, K, K.cpu(), 4),
                 lambda: G.sink_attention(q, K[:2], K[:2], 4), lambda: G.sink_attention(q, K[0], K[0], 4),
                 lambda: G.sink_attention(q, K.transpose(0, 1), K, 4),
                 lambda: G.sink_attention(q, K, K, 4, out=q.float())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: G.tree_attention(torch.zeros(4, 1, 65, 64, dtype=BF, device="cuda"), pg),
                 lambda: G.tree_attention(q, pg, window=-1),
                 lambda: G.tree_attention(q, pg, _i32([[-1] * 3] * 3)),
                 lambda: G.sink_attention(q, K[:, :2].contiguous(), K[:, :2].contiguous(), 4),
                 lambda: G.sink_attention(q, K, K, -1)):
        with pytest.raises(G.GrkvError):
            call()


# calls whose blocks hold 32 rows (many units of 17 to 64 rows), and splits of several row
# groups, joined (few) or combined (many): dtype, d, page, group, tokens, lens, units, window, sinks
ROW_CASES = [
    (BF, 128, 64, 5, 6, [6, 7, 40, 64, 65, 150, 333], 70, 0, 0),
    (BF, 64, 16, 8, 8, [8, 31, 100, 260], 36, 0, 0),
    (BF, 128, 32, 3, 7, [7, 90, 600], 66, 50, 6),
    (BF, 128, 64, 4, 8, [900, 1000, 8], 3, 0, 0),
    (BF, 64, 64, 4, 8, [4000, 5000, 700], 3, 0, 0),
    (F32, 128, 64, 4, 12, [1000, 300], 2, 0, 0),
    (F32, 64, 64, 2, 20, [3000, 30], 2, 0, 0),
]


@pytest.mark.parametrize("case", ROW_CASES, ids=lambda c: "%s-d%d-p%d-g%d-t%d-u%d-w%d" % (
    "bf16" if c[0] == BF else "f32", c[1], c[2], c[3], c[4], c[6], c[7]))
def test_row_groups_of_many_units_and_of_few(case):
    import paper_2605_31105_amd as G
    dtype, d, ps, group, t, lens, units, window, n_sink = case
    gen = torch.Generator().manual_seed(units + d)
    pg, K, V = _pool(lens, ps, d, dtype, gen)
    at = [e % len(lens) for e in range(units)]
    parents, plist = _parents("tree", 1, t, gen)
    q = torch.randn((units, group, t, d), generator=gen).to(dtype)
    o, lse = G.tree_attention(q.cuda(), pg, parents, units=_i32(at), window=window, n_sink=n_sink,
                              return_lse=True)
    again = G.tree_attention(q.cuda(), pg, parents, units=_i32(at), window=window, n_sink=n_sink)
    assert torch.equal(o, again)
    o, lse = o.cpu(), lse.cpu()
    for e in sorted({*range(len(lens)), *range(0, units, 11), units - 1}):
        u = at[e]
        for g in range(0, group, 2):
            check("entry %d" % e, o[e, g], lse[e, g], q[e, g], K[u], V[u],
                  tree_seen(lens[u], t, plist[0], window, n_sink))


def test_siblings_that_are_not_finite_in_calls_of_many_units():
    # a NaN and an infinity among the values of drafted token 2: only its own rows hold them
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(5)
    plist = [-1, 0, 0, 1, 2, 4, 3, 3]
    pg, K, V = _pool([70, 45], 16, 64, BF, gen)
    at = [e % 2 for e in range(64)]
    q = torch.randn((64, 3, 8, 64), generator=gen).to(BF)
    for unit, slot, value in ((0, 64, math.nan), (1, 39, math.inf)):
        pg.v[int(pg.table[unit, slot // 16]), slot % 16] = value
    o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, _i32([plist]), units=_i32(at), return_lse=True))
    for e in (0, 1, 30, 63):
        u = at[e]
        n = (70, 45)[u]
        seen = tree_seen(n, 8, plist, 0, 0)
        see = seen[:, (64, 39)[u]]
        assert see.any() and not see.all()
        for g in range(3):
            check("entry %d head %d" % (e, g), o[e, g, ~see], lse[e, g, ~see], q[e, g, ~see], K[u], V[u], seen[~see])
            assert not torch.isfinite(o[e, g, see]).any()


def test_prompts_of_few_rows_and_many_units():
    import paper_2605_31105_amd as G
    for dtype, U, group, nq, n, d, window in ((BF, 64, 4, 5, 77, 128, 0), (BF, 32, 4, 16, 300, 64, 40),
                                              (F32, 6, 4, 9, 500, 128, 0), (F32, 70, 3, 11, 64, 64, 9)):
        gen = torch.Generator().manual_seed(n)
        q = torch.randn((U, group, nq, d), generator=gen).to(dtype)
        K, V = (torch.randn((U, n, d), generator=gen).to(dtype) for _ in range(2))
        o, lse = (x.cpu() for x in G.sink_attention(q.cuda(), K.cuda(), V.cuda(), window, 3, return_lse=True))
        for u in (0, U // 2, U - 1):
            for g in range(group):
                check("unit %d head %d" % (u, g), o[u, g], lse[u, g], q[u, g], K[u], V[u],
                      sink_seen(n, nq, window, 3))


def test_two_captured_calls_share_a_workspace():
    # a call whose blocks join their splits, and one with a second launch: replayed in turn,
    # with an eager call of the same workspace and one that refills it between them
    import paper_2605_31105_amd as G
    gen = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn((3, 6000, 128), device="cuda", generator=gen).to(BF) for _ in range(2))
    qs = [torch.randn((3, 4, nq, 128), device="cuda", generator=gen).to(BF) for nq in (2, 12)]
    ws = torch.full((64 << 20,), 77, dtype=torch.uint8, device="cuda")
    want = [G.sink_attention(q, K, V, 0, return_lse=True) for q in qs]
    outs = [(torch.empty_like(o), torch.empty_like(l)) for o, l in want]
    graphs = []
    for q, (o, l) in zip(qs, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            G.sink_attention(q, K, V, 0, out=o, lse=l, workspace=ws)
    for k in range(6):
        for graph, (o, l), (wo, wl) in zip(graphs, outs, want):
            o.zero_()
            l.zero_()
            graph.replay()
            assert torch.equal(o, wo) and torch.equal(l, wl)
        eager = G.sink_attention(qs[k % 2], K, V, 0, workspace=ws)
        assert torch.equal(eager, want[k % 2][0])
        if k == 3:
            ws.fill_(3)


def test_workspaces_and_sizes_that_the_binding_refuses():
    import paper_2605_31105_amd as G
    pg = G.new_pages(4, 4, 8, 16, 64)
    q = torch.zeros(4, 2, 3, 64, dtype=BF, device="cuda")
    K = torch.zeros(4, 5, 64, dtype=BF, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    starts = torch.zeros(1, dtype=torch.int64, device="cuda")
    for call in (lambda: G.tree_attention(q, pg, workspace=ws),
                 lambda: G.sink_attention(q, K, K, 4, workspace=ws),
                 lambda: G.sink_attention(q, K, K, 4, workspace=ws.cuda()[::2]),
                 lambda: G.sink_attention(q, K, K, 4, workspace=ws.cuda()[:1].expand(1 << 16)),
                 lambda: G.pages_append(pg, K, K, workspace=ws),
                 lambda: G.sink_attention(q, K, K, 1 << 32), lambda: G.sink_attention(q, K, K, 4, 1 << 31),
                 lambda: G.tree_attention(q, pg, window=(1 << 32) + 5),
                 lambda: G.pages_append(pg, K[0], K[0], starts=starts, rows=1 << 32),
                 lambda: G.pages_compact(pg, _i32([0]), starts=starts, rows=(1 << 32) + 1)):
        with pytest.raises(ValueError):
            call()
    assert not pg.lens.any()


# calls of enough keys that they are cut into equal parts over the units: dtype, d, page, group,
# tokens, lens, entries, longest table row, window, sinks
EVEN_CASES = [
    (BF, 128, 64, 4, 1, [0, 1, 33, 2000, 640, 31, 900], 300, 32, 0, 0),
    (BF, 64, 16, 3, 5, [5, 0, 777, 1500, 6, 4], 420, 94, 0, 0),
    (BF, 128, 32, 8, 4, [4, 1100, 90, 2100], 280, 66, 0, 0),
    (BF, 128, 256, 1, 1, [0, 0, 1, 0], 4096, 2, 0, 0),
    (BF, 64, 64, 2, 7, [50, 3000, 200], 9, 1024, 40, 9),
    (BF, 128, 64, 4, 2, [60000, 70, 2], 5, 2048, 0, 0),
    (F32, 128, 16, 2, 3, [3, 400, 1000, 0], 270, 63, 0, 0),
    (F32, 64, 64, 5, 2, [2, 1234, 65], 250, 20, 300, 5),
    (BF, 128, 64, 4, 32, [32, 2000, 0, 700, 31], 240, 140, 0, 0),
    (BF, 64, 16, 2, 40, [41, 1500, 64, 90], 430, 94, 0, 0),
    (BF, 128, 128, 9, 14, [14, 33000, 400], 7, 2400, 0, 0),
    (BF, 128, 64, 4, 32, [32, 2000, 0, 700, 31], 240, 40, 300, 5),
    (BF, 64, 32, 5, 30, [1500, 0, 64], 5, 1000, 900, 40),
]


@pytest.mark.parametrize("case", EVEN_CASES, ids=lambda c: "%s-d%d-p%d-g%d-t%d-e%d-w%d" % (
    "bf16" if c[0] == BF else "f32", c[1], c[2], c[3], c[4], c[6], c[8]))
def test_units_of_any_lengths_in_equal_parts(case):
    import paper_2605_31105_amd as G
    dtype, d, ps, group, t, lens, entries, width, window, n_sink = case
    gen = torch.Generator().manual_seed(entries)
    pg, K, V = _pool(lens, ps, d, dtype, gen)
    table = torch.full((len(lens) + 1, width), -1, dtype=torch.int32, device="cuda")
    table[:, :pg.table.shape[1]] = pg.table[:, :width]
    pg = G.Pages(pg.k, pg.v, table, pg.lens, pg.refs, pg.free)
    at = torch.randint(len(lens), (entries,), generator=gen).tolist()
    counts = [t if k % 5 else k % (t + 1) for k in range(entries)]
    parents, plist = _parents("tree", 1, t, gen)
    q = torch.randn((entries, group, t, d), generator=gen).to(dtype)
    o = torch.full(q.shape, 5.0, dtype=dtype, device="cuda")
    lse = torch.full(q.shape[:3], 6.0, device="cuda")
    G.tree_attention(q.cuda(), pg, parents, units=_i32(at), counts=_i32(counts), window=window,
                     n_sink=n_sink, out=o, lse=lse)
    again = torch.full_like(o, 5.0)
    G.tree_attention(q.cuda(), pg, parents, units=_i32(at), counts=_i32(counts), window=window,
                     n_sink=n_sink, out=again)
    assert torch.equal(o, again)
    o, lse = o.cpu(), lse.cpu()
    for e in sorted({*range(0, entries, max(1, entries // 40)), entries - 1, entries - 2}):
        u, c = at[e], counts[e]
        assert (o[e, :, c:] == 5).all() and (lse[e, :, c:] == 6).all()
        for g in range(0, group, 2):
            check("entry %d" % e, o[e, g, :c], lse[e, g, :c], q[e, g, :c], K[u], V[u],
                  tree_seen(lens[u], c, plist[0], window, n_sink))


def test_equal_parts_captured_and_values_that_are_not_finite():
    # drafted token 2 of one unit holds a NaN; replays with other lengths than at the capture
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(8)
    lens, entries, plist = [1500, 300, 20], 360, [-1, 0, 0, 1]
    pg, K, V = _pool(lens, 64, 64, BF, gen)
    slot = 300 - 4 + 2
    pg.v[int(pg.table[1, slot // 64]), slot % 64, 7] = math.nan
    at = [e % 3 for e in range(entries)]
    q = torch.randn((entries, 2, 4, 64), generator=gen).to(BF)
    qd, units, parents = q.cuda(), _i32(at), _i32([plist])
    out, lse = torch.empty_like(qd), torch.empty(q.shape[:3], device="cuda")
    G.tree_attention(qd, pg, parents, units=units, out=out, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.tree_attention(qd, pg, parents, units=units, out=out, lse=lse)
    for held in (lens, [700, 300, 4], lens):
        pg.lens[:3] = _i32(held)
        out.zero_()
        graph.replay()
        eager, le = G.tree_attention(qd, pg, parents, units=units, return_lse=True)
        assert torch.equal(torch.nan_to_num(out, 9.0), torch.nan_to_num(eager, 9.0)) and torch.equal(lse, le)
        for e in (0, 1, 2, 178, 358, 359):
            u = at[e]
            n = held[u]
            seen = tree_seen(n, 4, plist, 0, 0)
            clean = ~seen[:, slot] if u == 1 else torch.ones(4, dtype=torch.bool)
            for g in range(2):
                check("entry %d" % e, eager[e, g].cpu()[clean], le[e, g].cpu()[clean], q[e, g, clean],
                      K[u][:n], V[u][:n], seen[clean])
                assert u != 1 or torch.isnan(eager[e, g, 2, 7]).item()


def _wide_table(pg, units, width):
    table = torch.full((units + 1, width), -1, dtype=torch.int32, device="cuda")
    table[:, :pg.table.shape[1]] = pg.table
    return __import__("paper_2605_31105_amd").Pages(pg.k, pg.v, table, pg.lens, pg.refs, pg.free)


@pytest.mark.parametrize("d,group,tokens,lens", [(64, 48, 6, [70, 6, 5]), (128, 16, 6, [90, 4000]),
                                                 (128, 5, 40, [41, 300, 39, 1200])])
def test_many_rows_and_siblings_that_are_not_finite(d, group, tokens, lens):
    # tables long enough that calls of these rows are the wide kernel's
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + tokens)
    pg, K, V = _pool(lens, 16, d, BF, gen)
    pg = _wide_table(pg, len(lens), 1200)
    assert len(lens) * group * tokens * 1200 * 16 > 1 << 20
    parents, plist = _parents("tree", 1, tokens, gen)
    q = torch.randn((len(lens), group, tokens, d), generator=gen).to(BF)
    for value in (None, math.nan, math.inf):
        where = [max(0, n - tokens) + 2 for n in lens]   # a drafted token of each unit
        for u, slot in enumerate(where):
            if value is not None:
                pg.v[int(pg.table[u, slot // 16]), slot % 16, 3:9] = value
        o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, parents, units=_i32(list(range(len(lens)))),
                                                    return_lse=True))
        for u, n in enumerate(lens):
            seen = tree_seen(n, tokens, plist[0], 0, 0)
            see = seen[:, where[u]] if value is not None else torch.zeros(tokens, dtype=torch.bool)
            for g in range(0, group, 5):
                check("unit %d head %d" % (u, g), o[u, g, ~see], lse[u, g, ~see], q[u, g, ~see], K[u], V[u], seen[~see])
                assert not torch.isfinite(o[u, g, see, 3:9]).any()


@pytest.mark.parametrize("d,window", [(64, 0), (128, 0), (128, 230)])
def test_prompts_of_many_rows_with_values_that_are_not_finite(d, window):
    # a NaN and an infinity among the values of keys 300 and 301: queries before them, and those
    # whose window has passed them, are the finite prompt's
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d + window)
    n, group = 700, 3
    q = torch.randn((2, group, n, d), generator=gen).to(BF)
    K, V = (torch.randn((2, n, d), generator=gen).to(BF) for _ in range(2))
    bad = V.clone()
    bad[:, 300, 5], bad[:, 301, 6] = math.nan, -math.inf
    assert 2 * group * n * (window + 48 if window else n) > 1 << 20   # (the wide kernel's)
    seen = sink_seen(n, n, window, 4)
    see = seen[:, 300] | seen[:, 301]
    for values in (V, bad):
        o, lse = (x.cpu() for x in G.sink_attention(q.cuda(), K.cuda(), values.cuda(), window, 4, return_lse=True))
        ok = ~see if values is bad else torch.ones(n, dtype=torch.bool)
        for u in range(2):
            for g in range(group):
                check("unit %d head %d" % (u, g), o[u, g, ok], lse[u, g, ok], q[u, g, ok], K[u], V[u], seen[ok])
        if values is bad:
            assert torch.isnan(o[:, :, seen[:, 300], 5]).all()
            assert not torch.isfinite(o[:, :, seen[:, 301], 6]).any()


def test_parents_without_a_tree_are_refused():
    # (an empty tensor has no address, which would say "a chain")
    import paper_2605_31105_amd as G
    pg = G.new_pages(4, 4, 8, 16, 64)
    q = torch.zeros(4, 2, 3, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        G.tree_attention(q, pg, torch.zeros((0, 3), dtype=torch.int32, device="cuda"))
