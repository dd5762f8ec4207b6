"""Refusals of the calls on pages, on the CPU: every bad argument is found on the host
before anything is launched."""
import ctypes

import pytest

import paper_2605_31105_amd as G

INV, UNS, WS = G.GRKV_ERR_INVALID, G.GRKV_ERR_UNSUPPORTED, G.GRKV_ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(G.lib_path()):
        pytest.skip("libgrkv.so not built")
    return G.lib()


def _pool(**kw):
    a = dict(k=4096, v=4096, table=4096, lens=4096, refs=4096, free_bits=4096, pages=100,
             page_size=64, units=8, max_pages=16, head_dim=128, dtype=0)
    a.update(kw)
    return G._PagesC(*a.values())


def _entries(**kw):
    a = dict(entries=4, units=4096, rows=3, counts=None, starts=None, source_rows=12, status=None)
    a.update(kw)
    return G._PageEntries(*a.values())


POOL = [(dict(k=None), INV), (dict(v=None), INV), (dict(table=None), INV), (dict(lens=None), INV),
        (dict(refs=None), INV), (dict(free_bits=None), INV), (dict(k=4104), INV), (dict(v=4100), INV),
        (dict(pages=0), INV), (dict(pages=(1 << 30) + 1), INV), (dict(units=0), INV),
        (dict(max_pages=0), INV), (dict(max_pages=1 << 25, page_size=64), INV),
        (dict(dtype=2), INV), (dict(page_size=8), UNS), (dict(page_size=48), UNS),
        (dict(page_size=2048), UNS), (dict(head_dim=96), UNS)]
ENTRIES = [(dict(entries=-1), INV), (dict(rows=-1), INV), (dict(source_rows=-1), INV),
           (dict(entries=1 << 20, rows=2048), INV)]


@pytest.mark.parametrize("kw,code", POOL)
def test_bad_pool(L, kw, code):
    pg, en, ws = _pool(**kw), _entries(), 1 << 30
    assert L.grkv_pages_workspace_bytes(pg, 4) == 0
    assert L.grkv_pages_init(pg, None) == code
    assert L.grkv_pages_append(pg, en, 4096, 0, 4096, 0, None, 4096, ws) == code
    assert L.grkv_pages_fork(pg, en, 4096, None, 4096, ws) == code
    assert L.grkv_pages_compact(pg, en, None, 4096, 4096, None, 4096, ws) == code
    assert L.grkv_pages_free(pg, en, None) == code


@pytest.mark.parametrize("kw,code", ENTRIES)
def test_bad_entries(L, kw, code):
    pg, en, ws = _pool(), _entries(**kw), 1 << 40
    assert L.grkv_pages_append(pg, en, 4096, 0, 4096, 0, None, 4096, ws) == code
    assert L.grkv_pages_compact(pg, en, None, 4096, 4096, None, 4096, ws) == code


def test_bad_calls(L):
    pg, en = _pool(), _entries()
    need = L.grkv_pages_workspace_bytes(pg, 4)
    assert need > 0 and need % 256 == 0 and L.grkv_pages_workspace_bytes(pg, -1) == 0
    for k, kt, v, vt, ws, size, code in [
            (None, 0, 4096, 0, 4096, need, INV), (4096, 0, None, 0, 4096, need, INV),
            (4104, 0, 4096, 0, 4096, need, INV), (4096, 2, 4096, 0, 4096, need, INV),
            (4096, 0, 4096, -1, 4096, need, INV), (4096, 0, 4096, 0, None, need, INV),
            (4096, 0, 4096, 0, 4096 + 16, need, INV), (4096, 0, 4096, 0, 4096, need - 1, WS)]:
        assert L.grkv_pages_append(pg, en, k, kt, v, vt, None, ws, size) == code
    assert L.grkv_pages_append(pg, None, 4096, 0, 4096, 0, None, 4096, need) == INV
    assert L.grkv_pages_fork(pg, en, None, None, 4096, need) == INV
    assert L.grkv_pages_fork(pg, en, 4096, None, 4096, need - 1) == WS
    assert L.grkv_pages_fork(pg, _entries(entries=1 << 25), 4096, None, 4096, 1 << 40) == INV
    assert L.grkv_pages_compact(pg, en, None, None, None, None, 4096, need) == INV
    assert L.grkv_pages_compact(pg, en, None, None, 4096, None, 4096, need - 1) == WS
    assert L.grkv_pages_free(pg, None, None) == INV


def test_calls_of_no_entries_do_nothing(L):
    # (no GPU here: a launch would fail)
    pg, en = _pool(), _entries(entries=0)
    assert L.grkv_pages_append(pg, en, None, 0, None, 0, None, None, 0) == 0
    assert L.grkv_pages_fork(pg, en, None, None, None, 0) == 0
    assert L.grkv_pages_compact(pg, en, None, None, None, None, None, 0) == 0
    assert L.grkv_pages_free(pg, en, None) == 0


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    i32 = dict(dtype=torch.int32)
    with pytest.raises(ValueError):
        G.Pages(k=torch.zeros(4, 16, 64), v=torch.zeros(4, 16, 64), table=torch.zeros((2, 2), **i32),
                lens=torch.zeros(2, **i32), refs=torch.zeros(4, **i32), free=torch.zeros(1, **i32))
    with pytest.raises(ValueError):
        G.new_pages(1, 1, 1, 16, 64, device="cpu")
    with pytest.raises(ValueError):
        G.new_pages(0, 1, 1, 16, 64, device="cpu")


def test_calls_of_more_entries_than_a_launch_has_blocks(L):
    # fork, compact and free are a block per entry, of 256 threads of a launch's 2^32: refused
    # on the host, before the plan changes the pool
    pg, ws = _pool(page_size=16), 1 << 40
    for n, code in (((1 << 24) - 1, WS), (1 << 24, INV), (3 << 24, INV)):
        en = _entries(entries=n, rows=1, source_rows=n)
        size = 256 if code == WS else ws   # (below the limit the workspace is what is refused)
        assert L.grkv_pages_fork(pg, en, 4096, None, 4096, size) == code
        assert L.grkv_pages_compact(pg, en, None, 4096, 4096, None, 4096, size) == code
        if code == INV:
            assert L.grkv_pages_free(pg, en, None) == code
    assert L.grkv_pages_append(pg, _entries(entries=1 << 25, rows=1, source_rows=1 << 25), 4096, 0, 4096, 0, None, 4096,
                               256) == WS


def test_sizes_past_32_bits_are_refused():
    # (ctypes would cut them, and ask for or work on another size)
    torch = pytest.importorskip("torch")

    class Pool:
        _c = _pool()

    class Tensor:
        def __init__(self, dtype, *shape):
            self.dtype, self.shape = dtype, torch.Size(shape)

        def dim(self):
            return len(self.shape)

        def get_device(self):
            return 0

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 4096

    def pool(units, width, pages):
        rows, i32 = (Tensor(torch.bfloat16, pages, 16, 64) for _ in range(2)), torch.int32
        return G.Pages(*rows, Tensor(i32, units, width), Tensor(i32, units), Tensor(i32, pages),
                       Tensor(i32, (pages + 31) // 32))

    big = 1 << 32
    assert pool(4, 3, 40)._c.units == 4
    for call in (lambda: pool(big + 4, 3, 40), lambda: pool(4, big + 3, 40), lambda: pool(4, 3, big + 40),
                 lambda: G.pages_workspace_bytes(Pool, big + 4),
                 lambda: G.tree_attention_workspace_bytes(Pool, big + 4, 1, 1),
                 lambda: G.tree_attention_workspace_bytes(Pool, 4, 1, 1, big),
                 lambda: G.sink_attention_workspace_bytes(big + 8, 4, 128, 0, 4096, 1, 0, 0),
                 lambda: G.sink_attention_workspace_bytes(8, 4, 128, 0, big + 4096, big + 1, 0, 0),
                 lambda: G.sink_attention_workspace_bytes(8, 4, 128, 0, 4096, 1, 0, big)):
        with pytest.raises(ValueError):
            call()
