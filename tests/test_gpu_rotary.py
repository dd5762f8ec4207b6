"""Rotary positions (rotary) and rows stored through a slot map (pages_store) against the
formulas in float64.

Bounds of a rotated column a cos x - b sin x (or a sin x + b cos x), all relative to s (|a| + |b|):
the reduced angle is rounded to float32 (2^-25), the series is cut below 2^-25 and summed in
float32 (2^-24 and a quarter of it inside), times s (2^-24, and 2^-24 of s itself), and the two
products are rounded once each (2 x 2^-24): 6.25 x 2^-24 in all, 2^-21 taken; p f and its
reduction in 64 bits are off by 4 x 2^-53 |p f|.  Then one rounding to the row's type."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _want(x, positions, freqs, scale, interleaved, inverse):
    """Rotated rows in float64, and their bounds before they are rounded to a type."""
    x, p, f = x.double().cpu(), positions.double().cpu(), freqs.double().cpu()
    r = 2 * f.numel()
    angle = (p[:, None] * f)[:, None]
    c, s = scale * torch.cos(angle), scale * torch.sin(angle)
    if inverse:
        s = -s
    y, tol = x.clone(), torch.zeros_like(x)
    ia, ib = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    tol[..., ia] = tol[..., ib] = abs(scale) * (a.abs() + b.abs()) * (2.0 ** -21 + 4 * 2.0 ** -53 * angle.abs())
    return y, tol


def _check(name, got, want, tol):
    half = 2.0 ** -8 if got.dtype == BF else 2.0 ** -24
    tol = tol + half * (want.abs() + tol)
    off = (got.double().cpu() - want).abs()
    worst = (off / tol.clamp(min=1e-300)).max().item() if off.numel() else 0.0
    print(name, "%.2f of the bound" % worst, flush=True)
    assert (off <= tol).all(), name


def _positions(n, far, gen):
    p = torch.randint(-far, far, (n,), generator=gen)
    p[:4] = torch.tensor([0, 1, far, -far])[:n]
    return p.to(torch.int32).cuda()


CASES = [
    # dtype, tokens, heads, columns, rotated, far
    (BF, 1, 1, 128, 128, 10), (BF, 3, 5, 64, 64, 131072), (BF, 257, 40, 128, 128, 1 << 20), (BF, 33, 3, 96, 48, 5000),
    (BF, 17, 2, 80, 36, 300), (BF, 9, 7, 2, 2, 100), (BF, 5, 3, 7, 4, 100), (BF, 1000, 1, 128, 64, (1 << 31) - 1),
    (BF, 2, 65, 256, 256, 77), (F32, 1, 32, 128, 128, 131072), (F32, 130, 6, 80, 36, 200000), (F32, 31, 3, 64, 32, 1 << 20),
    (F32, 8, 9, 6, 6, 50), (F32, 77, 2, 33, 18, 999), (F32, 4099, 2, 16, 8, 1 << 24), (BF, 20000, 9, 64, 64, 20000),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-t%d-h%d-d%d-r%d" % (("bf16" if c[0] == BF else "f32",) + c[1:5]))
def test_rotary(case, interleaved):
    import paper_2605_31105_amd as G
    dtype, T, H, d, r, far = case
    gen = torch.Generator().manual_seed(T + d + r)
    x = torch.randn((T, H, d), generator=gen).to(dtype).cuda()
    pos, f = _positions(T, far, gen), G.rotary_freqs(r, 1e4, device="cuda")
    for inverse, scale in ((False, 1.0), (True, 1.1386294)):
        y = G.rotary(x, pos, f, scale=scale, interleaved=interleaved, inverse=inverse)
        want, tol = _want(x, pos, f, scale, interleaved, inverse)
        _check("inverse %s" % inverse, y, want, tol)
        assert torch.equal(y[..., r:], x[..., r:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_places_and_layouts(interleaved):
    # heads before tokens, rows of a wider buffer, odd addresses, in place, into other strides
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(4)
    U, n, d = 3, 21, 64
    pos, f = _positions(n, 4000, gen), G.rotary_freqs(32, 1e4, device="cuda")
    base = torch.randn((U, n, d), generator=gen).to(BF).cuda()
    want, tol = _want(base.transpose(0, 1), pos, f, 1.0, interleaved, False)
    plain = G.rotary(base.transpose(0, 1).contiguous(), pos, f, interleaved=interleaved)
    _check("contiguous", plain, want, tol)
    assert torch.equal(G.rotary(base.transpose(0, 1), pos, f, interleaved=interleaved), plain)
    for lead in (0, 1, 8, 13):   # (an address that is no multiple of 16 bytes takes other loads, the same values)
        wide = torch.full((n, U, d + 24), 7.0, dtype=BF, device="cuda")
        view = wide[:, :, lead:lead + d]
        view.copy_(base.transpose(0, 1))
        out = torch.full((U, n, d + 3), 5.0, dtype=BF, device="cuda")
        got = G.rotary(view, pos, f, interleaved=interleaved, out=out.transpose(0, 1)[..., 1:d + 1])
        assert torch.equal(got, plain) and (out[..., 0] == 5).all() and (out[..., d + 1:] == 5).all()
        assert G.rotary(view, pos, f, interleaved=interleaved, out=view) is view
        assert torch.equal(view, plain)
        assert (wide[..., :lead] == 7).all() and (wide[..., lead + d:] == 7).all()
    one = base[0, :1, None].expand(1, 4, d)   # one row as four heads
    assert torch.equal(G.rotary(one, pos[:1], f, interleaved=interleaved)[:, 3], plain[:1, 0])


def test_rows_without_a_position_stay():
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(6)
    x = torch.randn((6, 2, 64), generator=gen).cuda()
    pos, f = _i32([3, G.NO_POSITION, 0, G.NO_POSITION, -2, 9]), G.rotary_freqs(64, device="cuda")
    out = torch.full_like(x, 5.0)
    G.rotary(x, pos, f, out=out)
    on = torch.tensor([0, 2, 4, 5])
    want, tol = _want(x[on], pos[on], f, 1.0, False, False)
    _check("rows", out[on], want, tol)
    assert (out[[1, 3]] == 5).all()
    assert G.rotary(x[:0], pos[:0], f).shape == (0, 2, 64) and G.rotary(x[:, :0], pos, f).shape == (6, 0, 64)


def test_values_that_are_not_finite_stay_in_their_pair():
    import paper_2605_31105_amd as G
    x = torch.ones((2, 1, 16), device="cuda")
    x[0, 0, 3], x[1, 0, 12] = math.nan, math.inf
    y = G.rotary(x, _i32([5, 5]), G.rotary_freqs(16, device="cuda"))
    bad = ~torch.isfinite(y[:, 0]).cpu()
    assert bad.nonzero().tolist() == [[0, 3], [0, 11], [1, 4], [1, 12]]


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_inverse_is_the_gradient(interleaved):
    # L = sum w y: dL/dx from the inverse against differences (the map is linear, so they are exact
    # but for float32's rounding of y: eight values of it, over steps of 1), and against autograd
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(8)
    x, w = torch.randn((3, 2, 8), generator=gen), torch.randn((3, 2, 8), generator=gen)
    pos, f, scale = _i32([0, 7, 5000]), G.rotary_freqs(6, device="cuda"), 1.25
    grad = G.rotary(w.cuda(), pos, f, scale=scale, interleaved=interleaved, inverse=True).cpu()

    def loss(v):
        return (G.rotary(v.cuda(), pos, f, scale=scale, interleaved=interleaved).cpu().double() * w).sum().item()

    size = (w.abs().sum() * scale * (x.abs().max() + 1) * 2).item()
    for at in [(0, 0, 0), (1, 1, 3), (2, 0, 5), (2, 1, 2), (1, 0, 7)]:
        up, down = x.clone(), x.clone()
        up[at] += 1
        down[at] -= 1
        assert abs((loss(up) - loss(down)) / 2 - grad[at].item()) <= 2.0 ** -20 * size
    v = x.double().requires_grad_()
    y, _ = _want(v.detach(), pos, f, scale, interleaved, False)
    angle = (pos.double().cpu()[:, None] * f.cpu())[:, None]
    c, s = scale * angle.cos(), scale * angle.sin()
    a, b = (v[..., :6:2], v[..., 1:6:2]) if interleaved else (v[..., :3], v[..., 3:6])
    parts = [a * c - b * s, a * s + b * c]
    wa, wb = (w[..., :6:2], w[..., 1:6:2]) if interleaved else (w[..., :3], w[..., 3:6])
    ((parts[0] * wa).sum() + (parts[1] * wb).sum() + (v[..., 6:] * w[..., 6:]).sum()).backward()
    _, tol = _want(w, pos, f, scale, interleaved, True)
    _check("gradient", grad, v.grad, tol)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_autograd_takes_the_inverse(dtype, interleaved):
    # bit for bit the call with `inverse`; rows without a position have no gradient, a sum's gradient
    # (one element as all) is taken, and the gradient has one of its own, the call again
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(18)
    x = torch.randn((9, 3, 80), generator=gen).to(dtype).cuda().requires_grad_()
    w = torch.randn((9, 3, 80), generator=gen).to(dtype).cuda()
    pos, f = _positions(9, 5000, gen), G.rotary_freqs(36, device="cuda")
    pos[5] = G.NO_POSITION
    on = torch.arange(9) != 5
    kw = dict(scale=1.25, interleaved=interleaved)
    for inverse in (False, True):
        y = G.rotary(x, pos, f, inverse=inverse, **kw)
        assert y.requires_grad and torch.equal(y[on], G.rotary(x.detach(), pos, f, inverse=inverse, **kw)[on])
        want = G.rotary(w, pos, f, inverse=not inverse, out=torch.zeros_like(w), **kw)
        for turn in range(2):
            got, = torch.autograd.grad(y, x, w, retain_graph=True)
            assert torch.equal(got, want) and not got[5].any()
        ones, = torch.autograd.grad(y[on].sum(), x, retain_graph=True)
        assert torch.equal(ones, G.rotary(torch.ones_like(w), pos, f, inverse=not inverse, out=torch.zeros_like(w), **kw))
        v = w.clone().requires_grad_()
        first, = torch.autograd.grad(y, x, v, create_graph=True)
        second, = torch.autograd.grad(first, v, w)
        assert torch.equal(second, G.rotary(w, pos, f, inverse=inverse, out=torch.zeros_like(w), **kw))
        all_of, = torch.autograd.grad(G.rotary(x, pos, f, inverse=inverse, **kw).sum(), x)
        assert torch.equal(all_of, ones)
    # strides and another stream; no gradient where none is asked for; an output of one's own has none
    side, z = torch.cuda.Stream(), x.detach().transpose(0, 1).contiguous().requires_grad_()
    side.wait_stream(torch.cuda.current_stream())
    y = G.rotary(z.transpose(0, 1), pos, f, stream=side, **kw)
    got, = torch.autograd.grad(y, z, w)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.transpose(0, 1), G.rotary(w, pos, f, inverse=True, out=torch.zeros_like(w), **kw))
    with torch.no_grad():
        assert not G.rotary(x, pos, f).requires_grad
        G.rotary(x, pos, f, out=torch.empty_like(x))
    for out in (x, torch.empty_like(x)):
        with pytest.raises(ValueError):
            G.rotary(x, pos, f, out=out)


def test_a_captured_gradient_is_replayed():
    # forward and backward in one graph, replayed with other rows and positions, eager calls between
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(28)
    x = torch.randn((33, 4, 64), generator=gen).cuda().requires_grad_()
    w, pos, f = torch.randn((33, 4, 64), generator=gen).cuda(), _positions(33, 900, gen), G.rotary_freqs(48, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(G.rotary(x, pos, f, scale=1.5), x, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = G.rotary(x, pos, f, scale=1.5)
        g, = torch.autograd.grad(y, x, w)
        y = y.detach()
    for turn in range(4):
        with torch.no_grad():
            x.copy_(torch.randn(x.shape, generator=gen))
            w.copy_(torch.randn(x.shape, generator=gen))
            pos.copy_(torch.randint(-50, 7000, (33,), generator=gen))
            pos[turn] = G.NO_POSITION
        graph.replay()
        torch.cuda.synchronize()
        on = torch.arange(33) != turn
        want, = torch.autograd.grad(G.rotary(x, pos, f, scale=1.5), x, w)
        assert torch.equal(g, want) and not g[turn].any()
        assert torch.equal(y[on], G.rotary(x.detach(), pos, f, scale=1.5)[on])


def test_there_and_back():
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(2)
    x = torch.randn((50, 3, 128), generator=gen).cuda()
    pos, f = _positions(50, 1 << 20, gen), G.rotary_freqs(128, device="cuda")
    y = G.rotary(G.rotary(x, pos, f), pos, f, inverse=True)
    # each way is within 2^-21 (|a| + |b|) of a rotation, by the bounds above, and rounds once
    tol = 2 * (2.0 ** -21 + 2.0 ** -24 + 4 * 2.0 ** -53 * 2.0 ** 20) * 2 * (x[..., :64].abs() + x[..., 64:].abs())
    off = (y - x).abs()
    assert (off <= torch.cat([tol, tol], -1)).all()


STORES = [
    # rows' type, pool's type, tokens, heads, group, d, rotated, page
    (BF, BF, 1, 8, 4, 128, 128, 64), (BF, BF, 100, 2, 1, 64, 64, 16), (BF, F32, 33, 3, 5, 128, 36, 16),
    (F32, BF, 64, 4, 2, 64, 32, 32), (F32, F32, 5, 1, 7, 128, 128, 1024), (BF, BF, 700, 8, 4, 128, 64, 64),
    (F32, BF, 9, 5, 1, 128, 2, 16), (BF, F32, 40, 2, 2, 64, 0, 16), (BF, BF, 12, 3, 0, 128, 128, 16),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", STORES, ids=lambda c: "%s-%s-t%d-h%d-g%d-d%d-r%d" % (
    ("bf16" if c[0] == BF else "f32", "bf16" if c[1] == BF else "f32") + c[2:7]))
def test_store(case, interleaved):
    import paper_2605_31105_amd as G
    dtype, ptype, T, H, group, d, r, ps = case
    gen = torch.Generator().manual_seed(T + d)
    pages = -(-(T * H) // ps) + 2
    pg = G.new_pages(H, 4, pages, ps, d, ptype)
    pg.k.fill_(5.0)
    pg.v.fill_(6.0)
    rows = torch.randn((T, H * group + 2 * H, d), generator=gen).to(dtype).cuda()
    q, k, v = rows.split([H * group, H, H], 1)
    slots = torch.randperm(pages * ps, generator=gen)[:T * H].view(T, H).cuda()
    pos = _positions(T, 100000, gen)
    if T > 4:   # rows that are no sequence's, and one without a slot
        slots[T - 1], pos[T - 1] = -1, G.NO_POSITION
        slots[2, 0] = -1
        if H > 1:
            slots[3, 1] = pages * ps   # (past the pool)
    out = torch.full((T, H * group, d), 7.0, dtype=dtype, device="cuda") if group and r else None
    if r:
        f = G.rotary_freqs(r, device="cuda")
        got = G.pages_store(pg, slots, k, v, q=q if group else None, positions=pos, freqs=f, scale=1.2,
                            interleaved=interleaved, out=out)
        kw, kt = _want(k, pos, f, 1.2, interleaved, False)
    else:
        got = G.pages_store(pg, slots, k, v)
        kw, kt = k.double().cpu(), torch.zeros(k.shape, dtype=torch.float64)
    assert got is out
    on = ((slots >= 0) & (slots < pages * ps)).cpu()
    at = slots.cpu()[on]
    K, V = pg.k.view(-1, d).cpu(), pg.v.view(-1, d).cpu()
    _check("keys", K[at], kw[on], kt[on])
    assert torch.equal(V[at], v.cpu()[on].to(ptype))
    rest = torch.ones(pages * ps, dtype=torch.bool)
    rest[at] = False
    assert (K[rest] == 5).all() and (V[rest] == 6).all()
    if out is not None:
        live = pos.cpu() != G.NO_POSITION
        qw, qt = _want(q, pos, f, 1.2, interleaved, False)
        _check("queries", out.cpu()[live], qw[live], qt[live])
        assert (out.cpu()[~live] == 7).all()


def test_store_of_a_layer_of_a_models_slots():
    # the columns of one layer, queries rotated in place, other streams, a captured call
    import paper_2605_31105_amd as G
    gen = torch.Generator().manual_seed(5)
    T, H, L, d, ps = 9, 2, 3, 64, 16
    pg = G.new_pages(1, 4, 8, ps, d, BF)
    every = torch.randperm(8 * ps, generator=gen)[:T * H * L].view(T, H * L).cuda()
    slots = every[:, H:2 * H]
    k, v, q = (torch.randn((T, n, d), generator=gen).to(BF).cuda() for n in (H, H, 4))
    pos, f = _positions(T, 999, gen), G.rotary_freqs(d, device="cuda")
    want_q, want_k = G.rotary(q, pos, f), G.rotary(k, pos, f)
    pg.k.zero_()
    q0 = q.clone()
    assert G.pages_store(pg, slots, k, v, q=q, positions=pos, freqs=f, out=q) is q
    assert torch.equal(q, want_q)
    assert torch.equal(pg.k.view(-1, d)[slots], want_k) and torch.equal(pg.v.view(-1, d)[slots], v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pg.k.zero_()
    side.wait_stream(torch.cuda.current_stream())
    out = G.pages_store(pg, slots, k, v, q=q0, positions=pos, freqs=f, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want_q) and torch.equal(pg.k.view(-1, d)[slots], want_k)
    graph = torch.cuda.CUDAGraph()
    out.zero_()
    y = torch.empty_like(q0)
    with torch.cuda.graph(graph):
        G.pages_store(pg, slots, k, v, q=q0, positions=pos, freqs=f, out=out)
        G.rotary(q0, pos, f, out=y)
    for turn in range(3):
        q0.copy_(torch.randn(q0.shape, generator=gen).to(BF))
        k.copy_(torch.randn(k.shape, generator=gen).to(BF))
        pos.add_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, G.rotary(q0, pos, f)) and torch.equal(y, out)
        assert torch.equal(pg.k.view(-1, d)[slots], G.rotary(k, pos, f))


def test_binding_checks():
    import paper_2605_31105_amd as G
    x, pos, f = torch.zeros((4, 2, 64), device="cuda"), _i32([0] * 4), G.rotary_freqs(64, device="cuda")
    pg = G.new_pages(2, 2, 4, 16, 64, F32)
    slots = torch.zeros((4, 2), dtype=torch.int64, device="cuda")
    bad = [
        lambda: G.rotary(x.cpu(), pos, f), lambda: G.rotary(x[0], pos, f), lambda: G.rotary(x.half(), pos, f),
        lambda: G.rotary(x.transpose(1, 2), pos, f), lambda: G.rotary(x, pos[:3], f), lambda: G.rotary(x, pos.long(), f),
        lambda: G.rotary(x, pos, f.float()), lambda: G.rotary(x, pos, f.cpu()), lambda: G.rotary(x, pos, f[::2]),
        lambda: G.rotary(x, pos, f, out=x[:3]), lambda: G.rotary(x, pos, f, out=x.to(BF)),
        lambda: G.rotary(x, pos, f, out=torch.zeros((1, 2, 64), device="cuda").expand(4, 2, 64)),
        lambda: G.rotary(x[:2], pos[:2], f, out=torch.as_strided(x, (2, 2, 64), (64, 128, 1))),
        lambda: G.pages_store(pg, slots, x, x[:3]), lambda: G.pages_store(pg, slots.int(), x, x),
        lambda: G.pages_store(pg, slots[:3], x, x), lambda: G.pages_store(pg, slots, x[..., :32], x[..., :32]),
        lambda: G.pages_store(pg, slots, x, x, q=x), lambda: G.pages_store(pg, slots, x, x, positions=pos),
        lambda: G.pages_store(pg, slots, x, x, freqs=f), lambda: G.pages_store(pg, slots, x, x.to(BF)),
        lambda: G.pages_store(pg, slots, x, x, q=x.to(BF), positions=pos, freqs=f),
        lambda: G.pages_store(pg, slots, x, x, out=x), lambda: G.pages_store(pg, slots.t().contiguous().t(), x, x),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("call %d was taken" % i)
    for call in (lambda: G.rotary(x[..., :32], pos, f), lambda: G.pages_store(pg, slots, x, x, positions=pos,
                                                                              freqs=G.rotary_freqs(66, device="cuda"))):
        with pytest.raises(G.GrkvError) as e:
            call()
        assert e.value.status == G.GRKV_ERR_INVALID
