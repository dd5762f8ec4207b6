"""Attention and pages whose rows lie past 2^31 elements and 2^32 bytes of their tensors."""
import pytest

from tests.attention_ref import check, sink_seen, tree_seen
from tests.test_gpu_attention import BF, F32, _i32

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype,group,tokens,window", [(BF, 4, 1, 0), (BF, 4, 8, 300), (BF, 40, 4, 0), (F32, 2, 3, 0)])
def test_pages_past_two_to_the_31_elements(dtype, group, tokens, window):
    # only the pool's last pages are free, so rows are stored, copied and read there
    import paper_2605_31105_amd as G
    ps, d, n, width = 1024, 128, 1500, 32
    pages = (1 << 31) // (ps * d) + 40
    pg = G.new_pages(4, width, pages, ps, d, dtype)
    assert pg.k.numel() > 1 << 31
    gen = torch.Generator().manual_seed(tokens)
    held = pages - 8
    pg.refs[:held] = 1
    bits = torch.zeros(-(-pages // 32), dtype=torch.int64)
    for p in range(held, pages):
        bits[p // 32] |= 1 << (p % 32)
    pg.free.copy_(torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32))
    K, V = ((torch.randn((2, n, d), generator=gen)).to(dtype) for _ in range(2))
    assert not G.pages_append(pg, K.cuda(), V.cuda()).any().item()
    assert not G.pages_fork(pg, _i32([1]), _i32([3])).any().item()
    assert pg.table[:4, :2].min().item() == -1 and pg.table.max().item() == held + 4
    E = 24
    at = [(0, 1, 3)[e % 3] for e in range(E)]
    q = torch.randn((E, group, tokens, d), generator=gen).to(dtype)
    o, lse = (x.cpu() for x in G.tree_attention(q.cuda(), pg, units=_i32(at), window=window, n_sink=3, return_lse=True))
    seen = tree_seen(n, tokens, list(range(-1, tokens - 1)), window, 3)
    for e in (0, 1, 2, E - 1):
        u = (0, 1, 1)[e % 3]
        for g in {0, group - 1}:
            check("entry %d" % e, o[e, g], lse[e, g], q[e, g], K[u], V[u], seen)


@pytest.mark.parametrize("nq,window", [(1, 0), (1, 500), (70, 500)])
def test_keys_past_two_to_the_31_elements(nq, window):
    import paper_2605_31105_amd as G
    U, n, d, group = 33, 1 << 19, 128, 4
    gen = torch.Generator().manual_seed(nq)
    K, V = (torch.zeros((U, n, d), dtype=BF, device="cuda") for _ in range(2))
    assert K.numel() > 1 << 31
    m = 2000   # (the other keys: equal logits of zero and values of zero)
    k, v = (torch.randn((m, d), generator=gen).to(BF) for _ in range(2))
    K[-1, -m:], V[-1, -m:] = k.cuda(), v.cuda()
    q = torch.randn((U, group, nq, d), generator=gen).to(BF)
    o, lse = (x[-1].cpu() for x in G.sink_attention(q.cuda(), K, V, window, 0, return_lse=True))
    if window:
        seen = sink_seen(m, nq, window, 0)
        for g in (0, group - 1):
            check("head %d" % g, o[g], lse[g], q[-1, g], k, v, seen)
    else:
        logits = q[-1, :, 0].double() @ k.double().t() / d ** 0.5
        total = logits.exp().sum(1) + (n - m)
        want = logits.exp() @ v.double() / total[:, None]
        # the sums run over n keys, the zeros' among them: within (n + 64) 2^-24 of sum p |v|
        size = logits.exp() @ v.double().abs() / total[:, None]
        tol = (n + 64) * 2.0 ** -24 * size + 2.0 ** -8 * want.abs()
        assert ((o[:, 0].double() - want).abs() <= tol).all()
        assert ((lse[:, 0].double() - total.log()).abs() <= (n + 64) * 2.0 ** -24).all()
