"""Waits of the paged attention kernels that expire, and calls that their workspace does not suit."""
import ctypes as C

import pytest
import torch

from tests import paged_testlib as P

pytestmark = pytest.mark.gpu

SITE_CODES = {601, 611, 612, 613, 614, 621, 622, 623, 624, 625, 631,
              701, 702, 703, 711, 712, 713, 714, 715, 716, 717, 718, 721, 722, 723, 724, 732, 733, 741, 742}


@pytest.fixture(scope="module")
def B():
    from paper_2605_26266_b200 import binding
    return binding


def _short_budget(B, lens, n, heads, d, calls):
    """Calls with a budget of two cycles until a wait expires; the last one's code and output, and the same call with the default budget."""
    cache, table = P.filled(B, lens, [n] * len(lens), 2, d, 64, torch.Generator().manual_seed(1))
    q = torch.randn(len(lens), heads, n, d, device="cuda").bfloat16()
    status, lengths = P.ints([0]), P.ints(lens)
    try:
        B.kvq_set_wait_budget_cycles(2)
        for _ in range(calls):
            short = B.kvq_paged_attn(cache, q, table, lengths, 0.1, status_word=status)
            torch.cuda.synchronize()                                  # the kernels came back by themselves
            if int(status):
                break
    finally:
        B.kvq_set_wait_budget_cycles(0)
    code = int(status)
    status.zero_()
    out = B.kvq_paged_attn(cache, q, table, lengths, 0.1, status_word=status)
    assert int(status) == 0
    P.assert_close(out, P.attention(cache, q, table, lengths, 0.1)[0])
    return code, short, out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,heads", [(1, 4), (4, 16), (16, 4), (100, 2), (700, 4)])
def test_with_a_budget_of_two_cycles_the_kernels_return(B, d, n, heads):
    """A wait that is not complete at its first poll gives up.  Nothing is left waiting, the context stays usable, and the same call with the default budget
    is right again.  A first poll can be long enough for every wait of a launch: then the answer is right."""
    code, short, out = _short_budget(B, [3000, 500], n, heads, d, 50)
    if code:
        assert code in SITE_CODES and B.kvq_status_word_result(code) == B.KVQ_ERR_TIMEOUT
    else:
        assert torch.equal(short, out)


@pytest.mark.parametrize("problems", [[(128, 16, 4), (128, 1, 8), (64, 16, 4)], [(128, 300, 2), (64, 300, 2)]])
def test_an_expired_wait_sets_the_status_word(B, problems):
    """Ranges of many tiles: of either kernel, some problem has a wait that is longer than a poll."""
    codes = [_short_budget(B, [90000, 70000, 500], n, heads, d, 50)[0] for d, n, heads in problems]
    assert any(codes) and all(c in SITE_CODES and B.kvq_status_word_result(c) == B.KVQ_ERR_TIMEOUT for c in codes if c), codes


@pytest.mark.parametrize("n", [1, 200])
def test_a_workspace_that_does_not_suit_is_refused(B, n):
    cache, table = P.filled(B, [300], [n], 2, 128, 64, torch.Generator().manual_seed(2))
    q = torch.randn(1, 4, n, 128, device="cuda").bfloat16()
    out, lengths = torch.full_like(q, 3.0), P.ints([300])
    seqs = B.kvq_paged_batch(1, table.shape[1], table.shape[1], table.data_ptr(), lengths.data_ptr(), None)
    need = B.kvq_paged_attn_workspace_bytes(cache, seqs, 4, n, 1)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    s = B.kvq_strides(*q.stride()[:3])
    call = lambda p, size: B.lib.kvq_paged_attn(C.byref(cache.desc), C.byref(seqs), None, q.data_ptr(), s, 4, n, out.data_ptr(), s, 0.1, 0, 1, None, p, size,
                                               None, None)
    assert call(None, 0) == B.KVQ_ERR_WORKSPACE and call(ws.data_ptr(), need - 1) == B.KVQ_ERR_WORKSPACE
    assert call(ws.data_ptr() + 128, need) == B.KVQ_ERR_ALIGNMENT
    torch.cuda.synchronize()
    assert bool((out == 3.0).all())
    # contents do not matter: the workspace full of what is no number
    ws.fill_(0xFF)
    torch.cuda.synchronize()
    assert call(ws.data_ptr(), need) == B.KVQ_OK
    torch.cuda.synchronize()
    P.assert_close(out, P.attention(cache, q, table, lengths, 0.1)[0])


def test_calls_through_ctypes_give_the_same_bytes(B, monkeypatch):
    cache, table = P.filled(B, [300, 7], [40, 40], 2, 128, 64, torch.Generator().manual_seed(3))
    q, k, v = (torch.randn(2, h, 40, 128, device="cuda").bfloat16() for h in (4, 2, 2))
    cos, sin = P.rope_tables(400, 64)
    kw = dict(cos=cos, sin=sin, interleaved=True, n_new=P.ints([40, 3]))
    res = []
    for plain in (True, False):
        if not plain:
            monkeypatch.setattr(B, "_paged_append_call", lambda *_: B._NOT_PLAIN)
            monkeypatch.setattr(B, "_paged_attn_call", lambda *_: B._NOT_PLAIN)
        mine = B.PagedCache(cache.desc.pages, 2, 128, 64, buffers=[b.clone() for b in cache.buffers])
        B.kvq_paged_append(mine, k, v, table, P.ints([300, 7]), **kw)
        lse = torch.empty(2, 4, 40, device="cuda")
        res.append([*mine.buffers, B.kvq_paged_attn(mine, q, table, P.ints([300, 7]), 0.1, lse=lse, **kw), lse])
    assert all(torch.equal(a, b) for a, b in zip(*res))
