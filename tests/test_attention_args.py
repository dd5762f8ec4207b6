"""Refusals of the attention calls on the CPU: every bad argument is found on the host
before anything is launched.  And the reference's masks by hand."""
import os

import pytest

import paper_2605_31105_amd as G

INV, UNS, WS = G.GRKV_ERR_INVALID, G.GRKV_ERR_UNSUPPORTED, G.GRKV_ERR_WORKSPACE


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


def _tree(**kw):
    a = dict(entries=8, group=4, tokens=3, units=None, counts=None, parents=None, trees=0, window=0,
             n_sink=4)
    a.update(kw)
    return G._Tree(*a.values())


TREES = [(dict(entries=-1), INV), (dict(group=0), INV), (dict(tokens=0), INV), (dict(window=-1), INV),
         (dict(n_sink=-1), INV), (dict(parents=4096, trees=0), INV), (dict(parents=4096, trees=3), INV),
         (dict(tokens=65), UNS), (dict(entries=1 << 30, group=1 << 10, tokens=64), INV),
         (dict(group=1 << 25, tokens=64), INV)]


@pytest.mark.parametrize("kw,code", TREES)
def test_bad_tree(L, kw, code):
    assert L.grkv_tree_attention(4096, _pool(), _tree(**kw), 4096, None, None, 4096, 1 << 40) == code
    assert L.grkv_tree_attention_workspace_bytes(_pool(), _tree(**kw)) == 0


@pytest.mark.parametrize("kw,code", [(dict(page_size=24), UNS), (dict(head_dim=80), UNS),
                                     (dict(table=None), INV), (dict(k=4100), INV), (dict(dtype=9), INV)])
def test_bad_pool(L, kw, code):
    assert L.grkv_tree_attention(4096, _pool(**kw), _tree(), 4096, None, None, 4096, 1 << 40) == code


def test_bad_tree_calls(L):
    pg, tr = _pool(), _tree()
    need = L.grkv_tree_attention_workspace_bytes(pg, tr)
    assert need > 256
    for q, o, lse, ws, size, code in [(None, 4096, None, 4096, need, INV), (4096, None, None, 4096, need, INV),
                                      (4104, 4096, None, 4096, need, INV), (4096, 4098, None, 4096, need, INV),
                                      (4096, 4096, 4097, 4096, need, INV), (4096, 4096, None, None, need, INV),
                                      (4096, 4096, None, 4100, need, INV),
                                      (4096, 4096, None, 4096, need - 1, WS)]:
        assert L.grkv_tree_attention(q, pg, tr, o, lse, None, ws, size) == code
    assert L.grkv_tree_attention(4096, pg, None, 4096, None, None, 4096, need) == INV
    # no entries: nothing to do (and no GPU here: a launch would fail)
    assert L.grkv_tree_attention(None, pg, _tree(entries=0), None, None, None, None, 0) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(nq=0), INV), (dict(nq=1001), INV), (dict(n=(1 << 30) + 1), INV), (dict(window=-1), INV),
    (dict(n_sink=-1), INV), (dict(units=0), INV), (dict(group=0), INV), (dict(dtype=3), INV),
    (dict(d=96), UNS), (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(o=None), INV),
    (dict(q=4100), INV), (dict(k=4100), INV), (dict(v=4100), INV), (dict(o=4100), INV),
    (dict(lse=4097), INV), (dict(ws=None), INV), (dict(ws=4097), INV), (dict(size=64), WS),
    (dict(units=1 << 20, group=64, n=1 << 20, nq=1 << 20), INV)])
def test_bad_sink_calls(L, kw, code):
    a = dict(q=4096, k=4096, v=4096, o=4096, lse=None, n=1000, nq=7, window=100, n_sink=4, units=2, group=4,
             d=128, dtype=0, ws=4096, size=1 << 40)
    a.update(kw)
    prob = G.Problem(a["units"], a["group"], a["d"], a["dtype"])
    assert L.grkv_sink_attention(a["q"], a["k"], a["v"], a["n"], a["nq"], a["window"], a["n_sink"], None,
                                 prob, a["o"], a["lse"], a["ws"], a["size"]) == code


def test_workspaces(L):
    # many units need no splits; few long ones do
    assert G.sink_attention_workspace_bytes(2048, 4, 128, 0, 4096, 1, 0, 0) == 256
    few = G.sink_attention_workspace_bytes(8, 4, 128, 0, 131072, 1, 0, 0)
    assert few > 256 and G.sink_attention_workspace_bytes(8, 4, 128, 0, 1 << 20, 1, 512, 4) < few
    assert G.sink_attention_workspace_bytes(8, 4, 96, 0, 4096, 1, 0, 0) == 0


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    q, K = torch.zeros(1, 2, 1, 64), torch.zeros(1, 8, 64)
    with pytest.raises(ValueError):
        G.sink_attention(q, K, K, 4)


def test_the_reference_masks_by_hand():
    torch = pytest.importorskip("torch")
    from tests.attention_ref import rows, sink_seen, tree_seen
    T, F = True, False
    # two cached slots, then a token, its two children, and a second root
    got = tree_seen(6, 4, [-1, 0, 0, -1], 0, 0)
    assert got.tolist() == [[T, T, T, F, F, F], [T, T, T, T, F, F], [T, T, T, F, T, F], [T, T, F, F, F, T]]
    # a window of two positions and one sink: the children (position 3) see positions 2, 3 and 0
    got = tree_seen(6, 4, [-1, 0, 0, -1], 2, 1)
    assert got.tolist() == [[T, T, T, F, F, F], [T, F, T, T, F, F], [T, F, T, F, T, F], [T, T, F, F, F, T]]
    # fewer slots than tokens: the first of them has none of its own
    assert tree_seen(1, 2, [-1, -1], 0, 0).tolist() == [[F], [T]]
    assert sink_seen(5, 2, 2, 1).tolist() == [[T, F, T, T, F], [T, F, F, T, T]]
    # one key seen: o is its value, lse its logit; none: -inf
    q, K = torch.eye(2, 64) * 8, torch.eye(2, 64)
    o, lse, _, _ = rows(q, K, K * 3, torch.tensor([[T, F], [F, F]]), False)
    assert o[0, 0] == 3 and not o[1].any() and abs(lse[0] - 1) < 1e-12 and lse[1] == float("-inf")


def test_calls_of_more_blocks_than_a_launch_has(L):
    # a launch has fewer than 2^32 threads, and a block 256: known from the sizes alone
    most = (1 << 24) - 8
    assert G.sink_attention_workspace_bytes(most, 1, 64, 0, 1, 1, 0, 0) == 256
    assert G.sink_attention_workspace_bytes(1 << 24, 1, 64, 0, 1, 1, 0, 0) == 0
    assert G.sink_attention_workspace_bytes(1 << 21, 1, 64, 1, 128, 128, 0, 0) == 0   # 8 row groups each
    pg = _pool()
    assert L.grkv_tree_attention_workspace_bytes(pg, _tree(entries=most, group=1)) == 256
    for kw in (dict(entries=1 << 24, group=1), dict(entries=1 << 22, group=64, tokens=8)):
        assert L.grkv_tree_attention_workspace_bytes(pg, _tree(**kw)) == 0
        assert L.grkv_tree_attention(4096, pg, _tree(**kw), 4096, None, None, 4096, 1 << 40) == INV
    prob = G.Problem(1 << 24, 1, 64, 0)
    assert L.grkv_sink_attention(4096, 4096, 4096, 1, 1, 0, 0, None, prob, 4096, None, 4096, 1 << 40) == INV


def test_binding_refuses_streams_of_another_device():
    # a call's stream is one of its tensors' device: any other would be left for that
    # device's current one
    torch = pytest.importorskip("torch")

    class Stream:
        cuda_stream, device = 4096, torch.device("cuda", 1)

    with pytest.raises(ValueError, match="stream"):
        G._on(0, Stream())
