"""A served model's step as its calls are used together, and calls at the ends of their ranges."""
import math

import pytest

from tests.attention_ref import check, sink_seen
from tests.test_gpu_attention import BF, F32, _i32, _pool
from tests.test_gpu_rotary import _check, _want

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _rows(pg, u):
    """The keys and values that unit u holds, on the host."""
    n, ps = int(pg.lens[u]), pg.k.shape[1]
    j = torch.arange(n, device="cuda")
    page = pg.table[u].long()[j // ps]
    return pg.k[page, j % ps].cpu(), pg.v[page, j % ps].cpu()


@pytest.mark.parametrize("d,window", [(128, 0), (64, 300)])
def test_compressed_caches_go_on_with_prompts_and_tokens(d, window):
    # two sequences, one of them compressed, take a chunk and then tokens one by one, positions
    # going on where the prompt ended; each unit's rows are what was stored, in order
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(d)
    H, group, n, w, c, ps = 2, 4, 600, 16, 128, 32
    freqs = G.rotary_freqs(d, 1e4, method="parts", factor=4.0, length=512, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    raw = torch.randn((H, n, d), generator=gen).to(BF).cuda()
    K = G.rotary(raw.transpose(0, 1), pos, freqs).transpose(0, 1).contiguous()
    V = torch.randn((H, n, d), generator=gen).to(BF).cuda()
    q_obs = torch.randn((H * group, w, d), generator=gen).to(BF).cuda()
    q_obs = G.rotary(q_obs.transpose(0, 1), pos[-w:], freqs).transpose(0, 1).contiguous().view(H, group, w, d)
    res = G.compress(q_obs, K, V, w, c, 7, 1e-2)
    pg = G.new_pages(2 * H, 40, 200, ps, d, BF)
    assert not G.pages_append(pg, res.k_out, res.v_out, units=_i32([0, 1])).any().item()
    held = [list(_rows(pg, u)) for u in range(2 * H)]
    assert all(len(held[u][0]) == (c if u < H else 0) for u in range(2 * H))
    seen = [n, 0]
    for turn, counts in enumerate([[70, 45], [1, 1], [0, 3], [1, 0], [40, 1]]):
        T = sum(counts) + 2
        rows = torch.randn((T, H * group + 2 * H, d), generator=gen).to(BF).cuda()
        q, k, v = rows.split([H * group, H, H], 1)
        step = G.pages_extend(pg, _i32(counts), T, heads=H, seen=_i32(seen))
        assert not step.status.any().item()
        qr = G.pages_store(pg, step.slots, k, v, q=q, positions=step.positions, freqs=freqs)
        o, lse = G.chunk_attention(qr, pg, step.starts, heads=H, longest=max(counts), window=window, n_sink=4,
                                   return_lse=True)
        t0 = 0
        for b, m in enumerate(counts):
            at = slice(t0, t0 + m)
            p = torch.arange(seen[b], seen[b] + m)
            assert step.positions[at].tolist() == p.tolist()
            want, tol = _want(q[at], p, freqs, 1.0, False, False)
            _check("queries", qr[at], want, tol)
            for h in range(H):
                u = b * H + h
                want, tol = _want(k[at], p, freqs, 1.0, False, False)
                Ku, Vu = _rows(pg, u)
                assert torch.equal(Ku[:len(held[u][0])], held[u][0]) and torch.equal(Vu[:len(held[u][1])], held[u][1])
                _check("keys", Ku[len(held[u][0]):], want[:, h], tol[:, h])
                assert torch.equal(Vu[len(held[u][1]):], v[at, h].cpu())
                held[u] = [Ku, Vu]
                for x in range(h * group, (h + 1) * group) if m else ():
                    check("turn %d unit %d" % (turn, u), o[at, x].cpu(), lse[at, x].cpu(), qr[at, x].cpu(), Ku, Vu,
                          sink_seen(len(Ku), m, window, 4))
            t0 += m
            seen[b] += m
    # taken back to the compressed cache, whose pages are then all that is held
    G.pages_compact(pg, keep=_i32([c, c, 0, 0]))
    assert pg.lens.tolist() == [c, c, 0, 0] and int((pg.refs > 0).sum()) == 2 * c // ps


@pytest.mark.parametrize("counts,d", [([1, 1, 1], 128), ([1, 30, 2], 64)])
def test_a_captured_step_is_replayed(counts, d):
    # one graph of a whole layer's step, replayed with other rows, beside the same calls made eagerly
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(3)
    B, H, group, ps, T = 3, 2, 4, 16, sum(counts) + 1
    freqs = G.rotary_freqs(d, device="cuda")
    lens = [300, 290, 5, 33, 1000, 1]
    pools = [_pool(lens, ps, d, BF, torch.Generator().manual_seed(4))[0] for _ in range(2)]
    for p in pools:   # (tables with room to grow, pages handed out as the tables say)
        p.k.nan_to_num_(0.0)
        p.v.nan_to_num_(0.0)
    grown = []
    for p in pools:
        g = G.new_pages(B * H, 80, 600, ps, d, BF)
        for u, n in enumerate(lens):
            K, V = _rows(p, u)
            G.pages_append(g, K.cuda()[None], V.cuda()[None], units=_i32([u]))
        grown.append(g)
    eager, pg = grown
    rows = torch.randn((T, H * group + 2 * H, d), generator=gen).to(BF).cuda()
    q, k, v = rows.split([H * group, H, H], 1)
    n, seen = _i32(counts), _i32([700, 10, 2000])
    step = G.Step(_i32([0] * (B + 1)), _i32([0] * T), torch.zeros((T, H), dtype=torch.int64, device="cuda"), _i32([0] * B))
    qr, o = torch.zeros((T, H * group, d), dtype=BF, device="cuda"), torch.zeros((T, H * group, d), dtype=BF, device="cuda")
    ws = torch.empty(max(G.pages_extend_workspace_bytes(pg, B, H, T),
                         G.chunk_attention_workspace_bytes(pg, B, H, T, group, max(counts))), dtype=torch.uint8,
                     device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.pages_extend(pg, n, T, heads=H, seen=seen, out=step, workspace=ws)
        G.pages_store(pg, step.slots, k, v, q=q, positions=step.positions, freqs=freqs, out=qr)
        G.chunk_attention(qr, pg, step.starts, heads=H, longest=max(counts), out=o, workspace=ws)
        seen.add_(n)
    first = seen.clone()
    for turn in range(5):
        rows.copy_(torch.randn(rows.shape, generator=gen).to(BF))
        ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        s = G.pages_extend(eager, n, T, heads=H, seen=first + turn * n)
        q2 = G.pages_store(eager, s.slots, k, v, q=q, positions=s.positions, freqs=freqs,
                           out=torch.zeros((T, H * group, d), dtype=BF, device="cuda"))
        o2 = G.chunk_attention(q2, eager, s.starts, heads=H, longest=max(counts), out=torch.zeros_like(o))
        assert not s.status.any().item()
        for x, y in ((step.slots, s.slots), (step.positions, s.positions), (qr, q2), (o, o2), (pg.lens, eager.lens),
                     (pg.table, eager.table), (pg.free, eager.free)):
            assert torch.equal(x, y), turn
        for u in range(B * H):
            for x, y in zip(_rows(pg, u), _rows(eager, u)):
                assert torch.equal(x, y)


def test_joined_calls_are_captured_and_share_a_workspace():
    # few units of few rows, whose blocks join their parts: lengths that change the number of parts
    # between the replays of two graphs over one workspace
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(19)
    H, group, d = 3, 4, 128
    pg, K, V = _pool([2000] * H, 16, d, BF, gen)
    pg.k.nan_to_num_(0.0)
    pg.v.nan_to_num_(0.0)
    qs = [torch.randn((2, H * group, d), generator=gen).to(BF).cuda() for _ in range(2)]
    starts = _i32([0, 2])
    ws = torch.empty(G.chunk_attention_workspace_bytes(pg, 1, H, 2, group), dtype=torch.uint8, device="cuda").random_(0, 255)
    outs, graphs = [torch.zeros_like(q) for q in qs], []
    for q, out in zip(qs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            G.chunk_attention(q, pg, starts, heads=H, out=out, workspace=ws)
        graphs.append(g)
    for n in (2000, 3, 700, 1999, 33, 1200):
        pg.lens[:H] = _i32([n, max(n - 500, 2), 2])
        for g in graphs + graphs:
            g.replay()
        torch.cuda.synchronize()
        for q, out in zip(qs, outs):
            for h in range(H):
                m = (n, max(n - 500, 2), 2)[h]
                x = h * group + 1
                o, lse = G.chunk_attention(q, pg, starts, heads=H, return_lse=True)
                assert torch.equal(o, out)
                check("%d unit %d" % (n, h), o[:, x].cpu(), lse[:, x].cpu(), q[:, x].cpu(), K[h][:m], V[h][:m],
                      sink_seen(m, 2, 0, 0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_past_two_to_the_31_elements(dtype):
    # only the pool's last pages are free, so a step grows, stores and reads there
    import paper_2605_31105_amd as G
    ps, d, width, H, group = 1024, 128, 8, 2, 4
    pages = (1 << 31) // (ps * d) + 40
    pg = G.new_pages(2 * H, width, pages, ps, d, dtype)
    assert pg.k.numel() > 1 << 31
    gen = torch.Generator().manual_seed(23)
    held = pages - 10
    pg.refs[:held] = 1
    bits = torch.zeros(-(-pages // 32), dtype=torch.int64)
    for p in range(held, pages):
        bits[p // 32] |= 1 << (p % 32)
    pg.free.copy_(torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32))
    counts, freqs = [1300, 1], G.rotary_freqs(d, device="cuda")
    T = sum(counts)
    rows = torch.randn((T, H * group + 2 * H, d), generator=gen).to(dtype).cuda()
    q, k, v = rows.split([H * group, H, H], 1)
    step = G.pages_extend(pg, _i32(counts), T, heads=H)
    assert not step.status.any().item() and int(step.slots.min()) >= held * ps
    qr = G.pages_store(pg, step.slots, k, v, q=q, positions=step.positions, freqs=freqs)
    o, lse = G.chunk_attention(qr, pg, step.starts, heads=H, return_lse=True)
    t0 = 0
    for b, m in enumerate(counts):
        at = slice(t0, t0 + m)
        for h in range(H):
            Ku, Vu = _rows(pg, b * H + h)
            assert torch.equal(Vu, v[at, h].cpu()) and torch.equal(Ku, G.rotary(k, step.positions, freqs)[at, h].cpu())
            x = h * group + 3
            check("unit %d" % (b * H + h), o[at, x].cpu(), lse[at, x].cpu(), qr[at, x].cpu(), Ku, Vu, sink_seen(m, m, 0, 0))
        t0 += m


def test_rotated_rows_past_two_to_the_31_elements():
    import paper_2605_31105_amd as G
    T, H, d = 66000, 256, 128
    x = torch.zeros((T, H, d), dtype=BF, device="cuda")
    assert x.numel() > 1 << 31
    gen = torch.Generator().manual_seed(29)
    last = torch.randn((5, H, d), generator=gen).to(BF)
    x[-5:] = last.cuda()
    pos, f = torch.arange(T, dtype=torch.int32, device="cuda"), G.rotary_freqs(d, device="cuda")
    y = G.rotary(x, pos, f, out=x)
    want, tol = _want(last, pos[-5:], f, 1.0, False, False)
    _check("last rows", y[-5:], want, tol)
    assert not y[:-5].any()


def test_two_streams_at_once():
    # calls on two streams, each with a pool and outputs of its own
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(31)
    H, group, d = 2, 4, 64
    work = []
    for _ in range(2):
        pg, _, _ = _pool([900, 40, 77, 3000], 32, d, BF, gen)
        q = torch.randn((50, H * group, d), generator=gen).to(BF).cuda()
        starts = _i32([0, 49, 50])
        work.append((pg, q, starts, G.chunk_attention(q, pg, starts, heads=H), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = []
    for _ in range(10):
        for pg, q, starts, _, s in work:
            outs.append(G.chunk_attention(q, pg, starts, heads=H, stream=s))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o, work[i % 2][3])


def test_streams_of_another_device_and_broken_sums():
    import paper_2605_31105_amd as G
    pg = G.new_pages(2, 2, 8, 16, 64)
    q, starts = torch.zeros((2, 2, 64), dtype=BF, device="cuda"), _i32([0, 1, 2])

    class Other:   # (as torch names a stream of a device that is not the pool's)
        cuda_stream, device = 0, torch.device("cuda", 1)

    for call in (lambda: G.chunk_attention(q, pg, starts, heads=1, stream=Other()),
                 lambda: G.pages_extend(pg, _i32([1]), 1, heads=1, stream=Other()),
                 lambda: G.rotary(q, _i32([0, 0]), G.rotary_freqs(64, device="cuda"), stream=Other()),
                 lambda: G.pages_store(pg, torch.zeros((2, 2), dtype=torch.int64, device="cuda"), q, q, stream=Other())):
        with pytest.raises(ValueError):
            call()
    # starts that fall or pass the rows: nothing outside the packed rows is read or written
    o, lse = torch.full_like(q, 5.0), torch.full((2, 2), 6.0, device="cuda")
    for bad in ([2, 0, 1], [-7, 3, -9], [1 << 30, -(1 << 30), 5], [0, 2 ** 31 - 1, 2]):
        G.chunk_attention(q, pg, _i32(bad), heads=1, out=o, lse=lse)
    torch.cuda.synchronize()
    assert not torch.isnan(o.float()).any() and math.isfinite(float(o.float().sum()))


@pytest.mark.parametrize("d,window", [(128, 50), (64, 33)])
def test_compressed_caches_go_on_under_a_window_that_hides_slots(d, window):
    # (units of 128 to 240 slots: all but the window and four sinks are out of sight)
    test_compressed_caches_go_on_with_prompts_and_tokens(d, window)
