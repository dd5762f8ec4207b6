"""Refusals of a step's calls on the CPU: every bad argument is found on the host before anything
is launched.  And the frequencies of rotary positions, which are formed there."""
import math
import os
import random

import pytest

import paper_2605_31105_amd as G

INV, UNS, WS = G.GRKV_ERR_INVALID, G.GRKV_ERR_UNSUPPORTED, G.GRKV_ERR_WORKSPACE
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(G.lib_path()):
        pytest.skip("libgrkv.so not built")
    return G.lib()


def _pool(**kw):
    a = dict(k=4096, v=4096, table=4096, lens=4096, refs=4096, free_bits=4096, pages=100,
             page_size=64, units=8, max_pages=16, head_dim=128, dtype=0)
    a.update(kw)
    return G._PagesC(*a.values())


def _step(**kw):
    a = dict(sequences=4, heads=2, units=None, unit_stride=0, tokens=10)
    a.update(kw)
    return G._StepC(*a.values())


def _chunk(**kw):
    a = dict(group=4, longest=10, window=0, n_sink=0)
    a.update(kw)
    return G._Chunk(*a.values())


def _rotation(**kw):
    a = dict(freqs=4096, dims=64, interleaved=0, inverse=0, scale=1.0)
    a.update(kw)
    return G._Rotation(*a.values())


POOLS = [(dict(k=None), INV), (dict(lens=None), INV), (dict(k=4104), INV), (dict(pages=0), INV),
         (dict(dtype=2), INV), (dict(page_size=48), UNS), (dict(head_dim=96), UNS)]
STEPS = [(dict(sequences=-1), INV), (dict(heads=0), INV), (dict(tokens=-1), INV), (dict(units=4096, unit_stride=1), INV),
         (dict(sequences=1 << 20, heads=16), INV), (dict(tokens=1 << 30, heads=2), INV)]
CHUNKS = [(dict(group=0), INV), (dict(longest=0), INV), (dict(window=-1), INV), (dict(n_sink=-1), INV),
          (dict(group=1 << 29), INV)]


@pytest.mark.parametrize("kw,code", POOLS)
def test_bad_pool(L, kw, code):
    pg, st, rows = _pool(**kw), _step(), G._Rows(4096, 128, 128)
    assert L.grkv_pages_extend(pg, st, 4096, None, 4096, 4096, 4096, None, None, 4096, BIG) == code
    assert L.grkv_pages_extend_workspace_bytes(pg, st) == 0
    assert L.grkv_pages_store(pg, 4, 2, 4096, 2, rows, rows, 0, None, None, 0, None, None, None) == code
    assert L.grkv_chunk_attention(4096, pg, st, 4096, _chunk(), 4096, None, None, 4096, BIG) == code
    assert L.grkv_chunk_attention_workspace_bytes(pg, st, _chunk()) == 0


@pytest.mark.parametrize("kw,code", STEPS)
def test_bad_step(L, kw, code):
    pg, st = _pool(), _step(**kw)
    assert L.grkv_pages_extend(pg, st, 4096, None, 4096, 4096, 4096, None, None, 4096, BIG) == code
    assert L.grkv_pages_extend_workspace_bytes(pg, st) == 0
    assert L.grkv_chunk_attention(4096, pg, st, 4096, _chunk(), 4096, None, None, 4096, BIG) == code
    assert L.grkv_chunk_attention_workspace_bytes(pg, st, _chunk()) == 0


@pytest.mark.parametrize("kw,code", CHUNKS)
def test_bad_chunk(L, kw, code):
    assert L.grkv_chunk_attention(4096, _pool(), _step(), 4096, _chunk(**kw), 4096, None, None, 4096, BIG) == code
    assert L.grkv_chunk_attention_workspace_bytes(_pool(), _step(), _chunk(**kw)) == 0


def test_bad_calls(L):
    pg, st, ch = _pool(), _step(), _chunk()
    need = L.grkv_pages_extend_workspace_bytes(pg, st)
    assert need > 0 and need % 256 == 0
    good = [pg, st, 4096, None, 4096, 4096, 4096, None, None, 4096, need]
    for at, value, code in [(1, None, INV), (2, None, INV), (4, None, INV), (5, None, INV), (6, None, INV),
                            (9, None, INV), (9, 4100, INV), (10, need - 1, WS)]:
        args = list(good)
        args[at] = value
        assert L.grkv_pages_extend(*args) == code, at
    assert L.grkv_pages_extend(pg, _step(sequences=0), None, None, None, None, None, None, None, None, 0) == 0
    need = L.grkv_chunk_attention_workspace_bytes(pg, st, ch)
    assert need > 0 and need % 256 == 0
    good = [4096, pg, st, 4096, ch, 4096, 4096, None, 4096, need]
    for at, value, code in [(0, None, INV), (0, 4104, INV), (2, None, INV), (3, None, INV), (4, None, INV),
                            (5, None, INV), (5, 4098, INV), (6, 4097, INV), (8, None, INV), (8, 4100, INV),
                            (9, need - 1, WS)]:
        args = list(good)
        args[at] = value
        assert L.grkv_chunk_attention(*args) == code, at
    # nothing to do (and no GPU here: a launch would fail)
    for kw in (dict(sequences=0), dict(tokens=0)):
        assert L.grkv_chunk_attention(None, pg, _step(**kw), None, ch, None, None, None, None, 0) == 0
    # units in rows of a wider matrix; the largest numbers of rows
    assert L.grkv_chunk_attention_workspace_bytes(pg, _step(units=4096, unit_stride=64), ch) > 0
    assert L.grkv_chunk_attention_workspace_bytes(pg, _step(heads=1, tokens=(1 << 28) - 1), ch) > 0
    assert L.grkv_chunk_attention_workspace_bytes(pg, _step(heads=1, tokens=1 << 28), ch) == 0
    # float32 rows come in tiles of 32: too many for a launch's index
    assert L.grkv_chunk_attention_workspace_bytes(_pool(dtype=1), _step(heads=1, tokens=(1 << 28) - 1), ch) == 0


ROTARY = [(dict(tokens=-1), INV), (dict(heads=-1), INV), (dict(heads=65536), INV), (dict(d=1), INV),
          (dict(d=32770), UNS), (dict(dtype=2), INV), (dict(tokens=1 << 24), INV), (dict(positions=None), INV),
          (dict(rot=None), INV), (dict(x=G._Rows(None, 1, 1)), INV), (dict(y=G._Rows(4097, 1, 1)), INV),
          (dict(x=None), INV), (dict(rot=_rotation(dims=0)), INV), (dict(rot=_rotation(dims=63)), INV),
          (dict(rot=_rotation(dims=130)), INV), (dict(rot=_rotation(freqs=None)), INV), (dict(rot=_rotation(freqs=4100)), INV),
          (dict(dtype=1, x=G._Rows(4098, 1, 1)), INV)]


@pytest.mark.parametrize("kw,code", ROTARY, ids=range(len(ROTARY)))
def test_bad_rotary(L, kw, code):
    a = dict(x=G._Rows(4096, 128, 128), y=G._Rows(4096, 128, 128), tokens=4, heads=1, d=128, dtype=0, positions=4096,
             rot=_rotation())
    a.update(kw)
    assert L.grkv_rotary(*a.values(), None) == code


def test_rotary_of_nothing(L):
    for tokens, heads in ((0, 3), (3, 0)):
        assert L.grkv_rotary(None, None, tokens, heads, 128, 0, None, None, None) == 0


STORE = [(dict(tokens=-1), INV), (dict(heads=-1), INV), (dict(heads=32764, stride=65536), INV), (dict(stride=1), INV),
         (dict(q_heads=-1), INV), (dict(q_heads=65536), INV), (dict(dtype=2), INV), (dict(slots=None), INV),
         (dict(k=None), INV), (dict(v=G._Rows(4097, 1, 1)), INV), (dict(q=None), INV), (dict(q_out=None), INV),
         (dict(positions=None), INV), (dict(rot=_rotation(dims=130)), INV), (dict(tokens=1 << 24), INV)]


@pytest.mark.parametrize("kw,code", STORE, ids=range(len(STORE)))
def test_bad_store(L, kw, code):
    r = G._Rows(4096, 1024, 128)
    a = dict(pages=_pool(), tokens=4, heads=2, slots=4096, stride=2, k=r, v=r, dtype=0, q=r, q_out=r, q_heads=8,
             positions=4096, rot=_rotation())
    a.update(kw)
    assert L.grkv_pages_store(*a.values(), None) == code


def test_store_of_nothing(L):
    assert L.grkv_pages_store(_pool(), 0, 2, None, 2, None, None, 0, None, None, 0, None, None, None) == 0
    # no heads, and no rotation, without which queries are not read
    assert L.grkv_pages_store(_pool(), 3, 0, None, 0, None, None, 0, None, None, 8, None, None, None) == 0


def test_frequencies():
    # closed forms, each within a few roundings of 64 bits (2^-50 of it)
    def same(got, want):
        assert len(got) == len(want) and all(abs(a - b) <= 2.0 ** -50 * abs(b) for a, b in zip(got.tolist(), want))

    r, s = 16, 4.0
    plain = [1e4 ** (-2.0 * i / r) for i in range(r // 2)]
    same(G.rotary_freqs(r), plain)
    same(G.rotary_freqs(r, method="linear", factor=s), [f / s for f in plain])
    base = G.rotary_freqs(r, method="base", factor=s)
    assert base[0] == 1.0
    same(base[-1:], [plain[-1] / s])          # the lowest frequency is divided by the factor
    same(base, [(1e4 * s ** (r / (r - 2))) ** (-2.0 * i / r) for i in range(r // 2)])
    same(G.rotary_freqs(2, method="base", factor=s), [1.0])
    parts = G.rotary_freqs(r, method="parts", factor=s, length=8192, low=1, high=32)
    for f, p in zip(plain, parts.tolist()):
        turns = 8192 * f / (2 * math.pi)
        if turns >= 32:
            assert abs(p - f) <= 2.0 ** -50 * f
        elif turns <= 1:
            assert abs(p - f / s) <= 2.0 ** -50 * f
        else:
            y = (turns - 1) / 31
            assert f / s < p < f and abs(p - ((1 - y) * f / s + y * f)) <= 2.0 ** -49 * f
    same(G.rotary_freqs(r, method="parts", factor=1.0, length=100), plain)
    assert G.rotary_freqs(r).device.type == "cpu"


@pytest.mark.parametrize("args", [(0,), (3,), (32770,), (8, 0.0), (8, -1.0), (8, math.nan), (8, math.inf)])
def test_bad_frequencies(args):
    with pytest.raises(G.GrkvError):
        G.rotary_freqs(*args)


@pytest.mark.parametrize("kw", [dict(method="linear", factor=0.5), dict(method="base", factor=math.nan),
                                dict(method="linear", factor=math.inf), dict(method="parts", factor=2.0),
                                dict(method="parts", factor=2.0, length=100, low=4, high=4),
                                dict(method="parts", factor=2.0, length=100, low=-1, high=4),
                                dict(method="parts", factor=2.0, length=math.inf),
                                dict(method="parts", factor=2.0, length=100, high=math.inf)])
def test_bad_scaling(kw):
    with pytest.raises(G.GrkvError):
        G.rotary_freqs(8, **kw)


@pytest.mark.parametrize("dims,base,kw", [
    (128, 1e300, dict(method="base", factor=1e10)),      # the scaled base passes 64 bits: pairs without a turn
    (4, 1e200, dict(method="base", factor=1e100)),       # base * factor^2
    (64, 5e-324, {}),                                    # the highest frequency does (10^(323.3 * 62 / 64))
    (64, 1e300, dict(method="linear", factor=1e300)),    # the lowest falls to zero
    (64, 1e300, dict(method="parts", factor=1e300, length=100.0)),
])
def test_frequencies_that_64_bits_do_not_hold_are_refused(dims, base, kw):
    with pytest.raises(G.GrkvError) as e:
        G.rotary_freqs(dims, base, **kw)
    assert e.value.status == INV


@pytest.mark.parametrize("dims,base,kw", [(128, 1e300, {}), (128, 1e-300, {}), (128, 1e200, dict(method="base", factor=1e100)),
                                          (2, 1e300, dict(method="base", factor=1e300)), (64, 1e4, dict(method="linear", factor=1e300))])
def test_far_frequencies_that_64_bits_hold(dims, base, kw):
    f = G.rotary_freqs(dims, base, **kw)
    assert all(0 < x < math.inf for x in f.tolist())


def test_an_unknown_scaling():
    with pytest.raises(ValueError):
        G.rotary_freqs(8, method="other")


def _sets(buf, view):
    at = (view.data_ptr() - buf.data_ptr()) // buf.element_size()
    T, H, d = view.shape
    a, b, _ = view.stride()
    return {at + t * a + h * b + c for t in range(T) for h in range(H) for c in range(d)}


def test_whether_an_output_overlaps_its_input():
    # views of one buffer against the sets of their elements, and their refusal as `out`
    torch = pytest.importorskip("torch")
    rng, counted = random.Random(5), [0, 0, 0]
    buf = torch.zeros(4000)
    for _ in range(4000):
        T, H, d = rng.choice([1, 2, 3, 7]), rng.choice([1, 2, 3, 5]), rng.choice([2, 3, 8])
        views, shared = [], rng.random() < 0.7
        for k in range(2):
            if k == 0 or not shared:
                inner = rng.choice([d, d, d + 1, 2 * d, 3 * d, 0])
                outer = rng.choice([H * inner, 2 * H * inner, 4 * d, d * T, H * inner + 2 * d, 1, 0])
                step = (outer, inner) if rng.random() < 0.7 else (inner, outer)
            views.append(torch.as_strided(buf, (T, H, d), step + (1,), rng.choice([0, 1, d, 3 * d, H * d, rng.randrange(300)])))
        x, y = views
        a, b = _sets(buf, x), _sets(buf, y)
        same = x.data_ptr() == y.data_ptr() and all(x.stride(i) == y.stride(i) for i in (0, 1) if x.shape[i] > 1)
        assert G._rows_meet(x, y) == (bool(a & b) and not same), (x.shape, x.stride(), y.stride(), x.storage_offset(), y.storage_offset())
        counted[2 if same else bool(a & b)] += 1
    assert min(counted) > 100, counted


def test_an_output_among_the_rows_of_its_input():
    torch = pytest.importorskip("torch")
    wide = torch.zeros((6, 8, 16))
    x = wide[:, :4]
    for out in (wide[:, 2:6], wide[:, 1:5], torch.as_strided(wide, (6, 4, 16), (128, 16, 1), 8)):
        with pytest.raises(ValueError):
            G._out_rows(x, out, "out", -1)
    for out in (wide[:, 4:], x, wide[:, :4], torch.zeros_like(x)):   # beside the input, in place, elsewhere
        assert G._out_rows(x, out, "out", -1)[0] is out
    ahead = torch.zeros((7, 4, 16))
    with pytest.raises(ValueError):   # a token on
        G._out_rows(ahead[:6], ahead[1:], "out", -1)
    none = wide[:0]
    assert G._out_rows(none, wide[:0], "out", -1)[0].shape == (0, 8, 16)
