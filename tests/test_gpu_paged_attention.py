"""kvq_paged_attn against its definition in 64 bits."""
import math

import pytest
import torch

from tests import paged_testlib as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2605_26266_b200 import binding
    return binding


def _run(B, lens, news, q_heads, kv_heads, d, page, causal=True, window=0, rope=0, interleaved=False, grid=False, seed=0, n=None,
         scale=None, spread=True, q_size=1.0):
    gen = torch.Generator().manual_seed(seed)
    cache, table = P.filled(B, lens, news, kv_heads, d, page, gen, spread)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    n = max(max(news), 1) if n is None else n
    q = (torch.randn(len(lens), q_heads, n, d, device="cuda", generator=g) * q_size).bfloat16()
    kw = dict(causal=causal, window=window)
    if rope:
        kw["cos"], kw["sin"] = P.rope_tables(max(a + m for a, m in zip(lens, news)) + 3, rope)
        kw["interleaved"] = interleaved
        if grid:
            kw["positions"] = torch.randint(0, kw["cos"].shape[0], (len(lens), n), device="cuda", generator=g, dtype=torch.int32)
    scale = d ** -0.5 if scale is None else scale
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    status = P.ints([0])
    out = torch.full_like(q, 9.0)
    got = B.kvq_paged_attn(cache, q, table, P.ints(lens), scale, n_new=P.ints(news), lse=lse, status_word=status, out=out, **kw)
    assert got is out and int(status) == 0
    want, want_lse = P.attention(cache, q, table, P.ints(lens), scale, P.ints(news), **kw)
    P.assert_close(out, want, lse, want_lse, f"{lens} {news} {q_heads}/{kv_heads} d{d} page {page} causal {causal} window {window}")
    again = B.kvq_paged_attn(cache, q, table, P.ints(lens), scale, n_new=P.ints(news), **kw)
    assert torch.equal(again, out)                                        # the same bits, with and without the log-sum-exp
    return cache, table, q, out, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("q_heads,kv_heads", [(2, 2), (8, 2), (7, 1)])
def test_single_tokens(B, d, page, q_heads, kv_heads):
    _run(B, [0, 1, 127, 128, 129, 1000, 3333], [1] * 7, q_heads, kv_heads, d, page, rope=d // 2, seed=page)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [2, 5, 16, 17, 40, 64, 65, 128, 129, 257])
def test_chunks(B, d, causal, n):
    _run(B, [0, 300, 777], [n, n, max(n // 2, 1)], 4, 2, d, 32, causal=causal, rope=d, seed=n)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16, 32])
@pytest.mark.parametrize("n", [1, 3, 70])
def test_groups_of_query_heads(B, group, n):
    _run(B, [500, 63], [n, n], 2 * group, 2, 128, 64, seed=group)


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 129, 1000, 10 ** 6, 2 ** 31 - 1, 2 ** 40])
@pytest.mark.parametrize("n", [1, 6, 200])
def test_windows(B, window, n):
    _run(B, [0, 700, 130], [n] * 3, 4, 2, 64, 16, window=window, seed=n)


@pytest.mark.parametrize("n", [1, 4, 100])
@pytest.mark.parametrize("causal", [True, False])
def test_sequences_without_tokens_and_rows_without_queries(B, n, causal):
    _, _, _, out, lse = _run(B, [0, 40, 0, 100, 0], [0, 0, 1, n, n], 4, 2, 128, 32, causal=causal, seed=n, n=n)
    assert not bool(out[:2].any()) and bool((lse[:2] == -math.inf).all())
    if n > 1:
        assert not bool(out[2, :, 1:].any())


def test_an_empty_batch_and_no_queries(B):
    cache = B.PagedCache(2, 2, 64, 16)
    for b, n in ((0, 3), (2, 0)):
        q = torch.zeros(b, 4, n, 64, device="cuda").bfloat16()
        out = B.kvq_paged_attn(cache, q, torch.zeros(b, 1, dtype=torch.int32, device="cuda"), P.ints([0] * b), 0.1)
        assert out.shape == q.shape
    q = torch.ones(2, 4, 3, 64, device="cuda").bfloat16()                                  # a table without columns
    out = B.kvq_paged_attn(cache, q, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), P.ints([0, 0]), 0.1, n_new=P.ints([0, 0]))
    assert not bool(out.any())


@pytest.mark.parametrize("d,rope,interleaved", [(128, 128, False), (128, 128, True), (128, 96, False), (64, 48, True), (64, 16, False)])
@pytest.mark.parametrize("n", [1, 150])
def test_rotations(B, d, rope, interleaved, n):
    _run(B, [40, 300], [n, n], 6, 2, d, 32, rope=rope, interleaved=interleaved, grid=True, seed=9)


@pytest.mark.parametrize("n", [1, 9, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_large_and_small_scores(B, n, d):
    """One key takes all of a row, or all keys the same share."""
    _run(B, [900], [n], 4, 2, d, 64, scale=3.0, q_size=0.25, seed=1)
    _run(B, [900], [n], 4, 2, d, 64, scale=1e-6, seed=2)
    _run(B, [900], [n], 4, 2, d, 64, scale=1.0, q_size=1e-3, seed=3)


@pytest.mark.parametrize("n", [1, 7, 200])
@pytest.mark.parametrize("low,high", [(-64, 20), (-30, 30), (0, 60)])
def test_scales_of_pages_far_apart(B, n, low, high):
    """Values of one page are nothing beside those of another, the page's keys are not: the weights have to come out of the same sum."""
    gen = torch.Generator().manual_seed(3)
    cache, table = P.filled(B, [256], [n], 2, 128, 64, gen)
    g = torch.Generator(device="cuda").manual_seed(4)
    e = torch.where(torch.rand(cache.views()["v_scale"].shape, device="cuda", generator=g) < 0.5, low, high)
    cache.views()["v_scale"].copy_((e + 127).to(torch.uint8))
    q = torch.randn(1, 4, n, 128, device="cuda", generator=g).bfloat16()
    lse = torch.empty(q.shape[:3], device="cuda")
    out = B.kvq_paged_attn(cache, q, table, P.ints([256]), 0.1, lse=lse)
    want, want_lse = P.attention(cache, q, table, P.ints([256]), 0.1)
    P.assert_close(out, want, lse, want_lse)


@pytest.mark.parametrize("n", [1, 5, 140])
def test_a_nan_reaches_those_who_see_it(B, n):
    gen = torch.Generator().manual_seed(5)
    cache, table = P.filled(B, [100], [n], 2, 128, 32, gen)
    q = torch.randn(1, 4, n, 128, device="cuda").bfloat16()
    clean = B.kvq_paged_attn(cache, q, table, P.ints([100]), 0.1)
    at = 100 + n // 2
    page, slot = int(table[0, at // 32]), at % 32
    cache.buffers[0].view(-1, 2, 32, 128)[page, 1, slot, 17] = 0x7F                        # a key of head 1
    out = B.kvq_paged_attn(cache, q, table, P.ints([100]), 0.1)
    assert torch.equal(out[:, :2], clean[:, :2])                                           # query heads 0 and 1 have key head 0
    assert torch.equal(out[:, 2:, :n // 2], clean[:, 2:, :n // 2]) and bool(out[:, 2:, n // 2:].isnan().all())


@pytest.mark.parametrize("n", [1, 3, 33, 260])
def test_strides(B, n):
    gen, g = torch.Generator().manual_seed(6), torch.Generator(device="cuda").manual_seed(7)
    lens = [130, 9]
    cache, table = P.filled(B, lens, [n, n], 2, 64, 16, gen)
    x = torch.randn(2, n, 3, 6, 64, device="cuda", generator=g).bfloat16()                # [batch, tokens, (q, k, v), heads, d]
    q = x[:, :, 0].transpose(1, 2)
    room = torch.full((2, n, 6, 80), 5.0, device="cuda").bfloat16()
    out = room[..., 8:72].transpose(1, 2)
    wide = torch.full((2, table.shape[1] + 5), 7, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + table.shape[1]] = table
    table = wide[:, 2:2 + table.shape[1]]
    B.kvq_paged_attn(cache, q, table, P.ints(lens), 0.125, out=out)
    P.assert_close(out, P.attention(cache, q, table, P.ints(lens), 0.125)[0])
    assert bool((room[..., :8] == 5).all()) and bool((room[..., 72:] == 5).all())
    shared = q[:1, :1].expand(2, 6, n, 64)                                                # one query for all
    out = B.kvq_paged_attn(cache, shared, table, P.ints(lens), 0.125)
    P.assert_close(out, P.attention(cache, shared, table, P.ints(lens), 0.125)[0])


@pytest.mark.parametrize("n", [1, 2, 100, 600])
def test_what_has_been_appended_is_seen(B, n):
    """Append and attention together, on a stream of their own and from a graph: prompts, then tokens one by one."""
    g = torch.Generator(device="cuda").manual_seed(8)
    lens, hq, hk, d, page = [0, 37], 8, 2, 128, 64
    table, pages = P.make_table(lens, [n + 3] * 2, page, torch.Generator().manual_seed(9))
    cache = B.PagedCache(pages, hk, d, page)
    cos, sin = P.rope_tables(1000, d)
    lengths = P.ints([0, 0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        first = [torch.randn(2, h, 37, d, device="cuda", generator=g).bfloat16() for h in (hk, hk)]
        B.kvq_paged_append(cache, *first, table, lengths, n_new=P.ints(lens), cos=cos, sin=sin)
        lengths = P.ints(lens)
        for m in (n, 1, 1):
            q, k, v = (torch.randn(2, h, m, d, device="cuda", generator=g).bfloat16() for h in (hq, hk, hk))
            B.kvq_paged_append(cache, k, v, table, lengths, cos=cos, sin=sin)
            out = B.kvq_paged_attn(cache, q, table, lengths, d ** -0.5, cos=cos, sin=sin)
            P.assert_close(out, P.attention(cache, q, table, lengths, d ** -0.5, cos=cos, sin=sin)[0])
            lengths = lengths + m
    s.synchronize()
    lengths = lengths - 1                                                                 # the last step again, from a graph
    graph, kept = torch.cuda.CUDAGraph(), out.clone()
    with torch.cuda.graph(graph):
        B.kvq_paged_append(cache, k, v, table, lengths, cos=cos, sin=sin)
        out = B.kvq_paged_attn(cache, q, table, lengths, d ** -0.5, cos=cos, sin=sin)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, kept)


def test_random_shapes(B):
    import random
    rng = random.Random(12)
    for i in range(24):
        batch, page = rng.choice((1, 2, 7)), rng.choice((16, 32, 64, 128))
        lens = [rng.choice((0, rng.randint(0, 200), rng.randint(0, 5000))) for _ in range(batch)]
        top = rng.choice((1, 4, 30, 500))
        news = [rng.randint(0, top) for _ in range(batch)]
        kv = rng.choice((1, 2, 5))
        causal = rng.random() < 0.7
        _run(B, lens, news, kv * rng.choice((1, 2, 4, 6)), kv, rng.choice((64, 128)), page, causal=causal,
             window=rng.choice((0, rng.randint(1, 800))) if causal else 0, rope=rng.choice((0, 16, 64)), interleaved=rng.random() < 0.5,
             grid=rng.random() < 0.5, seed=200 + i, n=max(max(news), 1))


@pytest.mark.parametrize("n", [1, 200])
def test_faults_of_the_lists_are_reported(B, n):
    gen = torch.Generator().manual_seed(10)
    cache, table = P.filled(B, [150], [n], 2, 128, 32, gen)
    q = torch.randn(1, 4, n, 128, device="cuda").bfloat16()
    for entry in (-1, cache.desc.pages, 2 ** 31 - 1):
        bad = table.clone()
        bad[0, 1] = entry                                                                 # tokens 32 to 63 are not seen
        status = P.ints([0])
        out = B.kvq_paged_attn(cache, q, bad, P.ints([150]), 0.1, status_word=status)
        assert int(status) == B.KVQ_PAGED_BAD_PAGE
        gone = B.PagedCache(cache.desc.pages, 2, 128, 32, buffers=[b.clone() for b in cache.buffers])
        # a page whose keys lose against all others: the same as one that is not there
        gone.views()["k_codes"][int(table[0, 1])] = 0
        want = _without(gone, q, table, [150], 0.1, 32, 64)
        P.assert_close(out, want)
    for lengths, code in ((-5, B.KVQ_PAGED_BAD_LENGTH), (32 * table.shape[1], B.KVQ_PAGED_BAD_LENGTH), (2 ** 31 - 1, B.KVQ_PAGED_BAD_LENGTH)):
        status = P.ints([0])
        out = B.kvq_paged_attn(cache, q, table, P.ints([lengths]), 0.1, status_word=status)
        assert int(status) == code and bool(torch.isfinite(out).all())
    cos, sin = P.rope_tables(16, 128)
    status = P.ints([0])
    B.kvq_paged_attn(cache, q, table, P.ints([150]), 0.1, cos=cos, sin=sin, status_word=status)
    assert int(status) == B.KVQ_PAGED_BAD_POSITION


def _without(cache, q, table, lens, scale, lo, hi):
    """Attention that does not see tokens [lo, hi)."""
    v, d = cache.views(), cache.desc
    ids = table[0].long()
    n = q.shape[2]
    total = lens[0] + n
    k, val = ((v[x + "_codes"][ids].double() * torch.exp2(v[x + "_scale"][ids].double() - 127)[..., None, None])
              .transpose(0, 1).reshape(d.kv_heads, -1, d.head_dim)[:, :total] for x in "kv")
    j, at = torch.arange(total, device="cuda"), lens[0] + torch.arange(n, device="cuda")[:, None]
    sees = (j <= at) & ((j < lo) | (j >= hi))
    g = q.shape[1] // d.kv_heads
    s = torch.einsum("hnd,hkd->hnk", q[0].double(), k.repeat_interleave(g, 0)) * scale
    w = torch.softmax(s.masked_fill(~sees, -math.inf), -1)
    return torch.einsum("hnk,hkd->hnd", w, val.repeat_interleave(g, 0))[None]


@pytest.mark.parametrize("n", [1, 130])
def test_offsets_beyond_32_bits(B, n):
    pages = 300_000                                                                       # 128 * 128 * 300 000 = 4.9e9 bytes of codes, twice
    cache = B.PagedCache(pages, 1, 128, 128)
    gen = torch.Generator().manual_seed(13)
    small, table = P.filled(B, [400], [n], 1, 128, 128, gen)
    for x, y in zip(cache.buffers, small.buffers):
        x[-y.numel():] = y
    q = torch.randn(1, 4, n, 128, device="cuda").bfloat16()
    far = torch.where(table < small.desc.pages, table + (pages - small.desc.pages), table).to(torch.int32)
    a = B.kvq_paged_attn(cache, q, far, P.ints([400]), 0.1)
    assert torch.equal(a, B.kvq_paged_attn(small, q, table, P.ints([400]), 0.1))


@pytest.mark.parametrize("lens,n,hq,hk,d", [([70000], 1, 4, 1, 128), ([40000], 1, 8, 8, 64), ([20000, 3, 9000], 3, 4, 2, 128), ([30000], 40, 4, 2, 128),
                                            ([2000], 1500, 2, 1, 128), ([25000], 300, 2, 2, 64)])
def test_long_sequences(B, lens, n, hq, hk, d):
    _run(B, lens, [n] * len(lens), hq, hk, d, 64, rope=d, seed=77)


def test_many_sequences(B):
    lens = [(37 * i * i) % 1500 for i in range(300)]
    _run(B, lens, [1] * 300, 4, 2, 64, 16, seed=14)
    _run(B, lens[:60], [1 + i % 9 for i in range(60)], 8, 2, 128, 64, window=300, seed=15)
