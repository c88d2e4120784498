"""kvq_paged_append against its definition, code by code and scale by scale."""
import pytest
import torch

from tests import paged_testlib as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2605_26266_b200 import binding
    return binding


def _kv(b, h, n, d, gen, scale=1.0):
    k, v = (torch.randn(b, h, n, d, device="cuda", generator=gen) * scale for _ in range(2))
    k[..., 3] *= 20.0
    return k.bfloat16(), v.bfloat16()


def _run(B, lens, news, kv_heads, d, page, rope=0, interleaved=False, grid=False, seed=0, n=None):
    gen = torch.Generator().manual_seed(seed)
    cache, table = P.filled(B, lens, news, kv_heads, d, page, gen)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    n = max(news) if n is None else n
    k, v = _kv(len(lens), kv_heads, n, d, g)
    kw = {}
    if rope:
        kw["cos"], kw["sin"] = P.rope_tables(max(a + m for a, m in zip(lens, news)) + 3, rope)
        kw["interleaved"] = interleaved
        if grid:
            kw["positions"] = torch.randint(0, kw["cos"].shape[0], (len(lens), n), device="cuda", generator=g, dtype=torch.int32)
    ref = P.Reference(cache)
    status = P.ints([0])
    B.kvq_paged_append(cache, k, v, table, P.ints(lens), n_new=P.ints(news), status_word=status, **kw)
    ref.append(k, v, table, P.ints(lens), P.ints(news), **kw)
    ref.assert_same(cache)
    assert int(status) == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("rope,interleaved", [(0, False), (64, False), (64, True), (16, False), (16, True)])
def test_blocks_of_every_page_size(B, d, page, rope, interleaved):
    _run(B, [0, 5, page, 3 * page - 1, 200], [1, 2 * page, page + 7, 1, 131], 3, d, page, rope, interleaved, seed=page + d)


@pytest.mark.parametrize("lens,news", [([0], [1]), ([0], [0]), ([15], [1]), ([16], [1]), ([17, 0, 4], [0, 3, 0]), ([0] * 40, [1] * 40),
                                       ([1000], [777]), ([63, 64, 65], [65, 64, 63])])
def test_lengths(B, lens, news):
    _run(B, lens, news, 2, 128, 64, 128, seed=len(lens), n=max(max(news), 1))


@pytest.mark.parametrize("d,rope,interleaved", [(128, 128, False), (128, 128, True), (128, 96, False), (64, 48, True)])
def test_positions_of_their_own(B, d, rope, interleaved):
    _run(B, [40, 0], [300, 123], 4, d, 32, rope, interleaved, grid=True, seed=9)


def test_the_same_tokens_in_one_call_or_many(B):
    """Later tokens raise the scales of pages that earlier calls have begun."""
    gen, g = torch.Generator().manual_seed(1), torch.Generator(device="cuda").manual_seed(2)
    table, pages = P.make_table([0], [150], 64, gen)
    k, v = _kv(1, 2, 150, 128, g)
    k *= torch.linspace(0.01, 30.0, 150, device="cuda")[:, None].bfloat16()
    cache = B.PagedCache(pages, 2, 128, 64)
    ref = P.Reference(cache)
    at = 0
    for n in (1, 1, 30, 33, 1, 50, 34):
        part = k[:, :, at:at + n], v[:, :, at:at + n]                     # slices: strides of the whole tensor
        B.kvq_paged_append(cache, *part, table, P.ints([at]))
        ref.append(*part, table, P.ints([at]))
        at += n
    assert at == 150
    ref.assert_same(cache)
    whole = B.PagedCache(pages, 2, 128, 64)
    B.kvq_paged_append(whole, k, v, table, P.ints([0]))
    a, w = cache.views(), whole.views()
    for x in ("k_scale", "v_scale"):
        assert torch.equal(a[x], w[x])
    # a code that was moved is that of one rounding, but in the subnormal range, where it may be one step (2^-9) off
    assert float((a["k_codes"].float() - w["k_codes"].float()).abs().max()) <= 2.0 ** -9


def test_strides_and_repeated_calls(B):
    gen, g = torch.Generator().manual_seed(3), torch.Generator(device="cuda").manual_seed(4)
    lens, news = [10, 70], [45, 20]
    cache, table = P.filled(B, lens, news, 2, 64, 32, gen)
    x = torch.randn(2, 45, 3, 2, 64, device="cuda", generator=g).bfloat16()             # a projection's [batch, tokens, (q, k, v), heads, d]
    k, v = x[:, :, 1].transpose(1, 2), x[:, :, 2].transpose(1, 2).contiguous()
    wide = torch.full((2, table.shape[1] + 5), 7, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + table.shape[1]] = table
    table = wide[:, 2:2 + table.shape[1]]
    ref = P.Reference(cache)
    for _ in range(2):                                                                  # the second call writes what the first one has
        B.kvq_paged_append(cache, k, v, table, P.ints(lens), n_new=P.ints(news))
    ref.append(k, v, table, P.ints(lens), P.ints(news))
    ref.assert_same(cache)


def test_zeros_extremes_and_what_is_no_number(B):
    table = P.ints([[2, 0]])
    cache = B.PagedCache(3, 2, 64, 16)
    k, v = torch.zeros(1, 2, 20, 64, device="cuda").bfloat16(), torch.zeros(1, 2, 20, 64, device="cuda").bfloat16()
    k[0, 0, 3, 5], k[0, 0, 4, 6], k[0, 0, 5, 7] = float("inf"), -float("inf"), 3.0e38
    k[0, 1, 2, 9] = float("nan")
    v[0, 0, 1, 1], v[0, 0, 1, 2], v[0, 0, 6, 3] = float("nan"), 2.0, float("inf")
    v[0, 1, 17, 0], v[0, 1, 18, 0] = 1e-38, 1e-25
    k[0, 1, 18, 2] = 448.0
    k[0, 1, 19, 2] = -1.75 * 2.0 ** -3
    ref = P.Reference(cache)
    B.kvq_paged_append(cache, k, v, table, P.ints([0]))
    ref.append(k, v, table, P.ints([0]))
    ref.assert_same(cache)
    codes = cache.views()["k_codes"].float()
    assert codes[2, 0, 3, 5] == 448 and codes[2, 0, 4, 6] == -448 and bool(codes[2, 0, 1].isnan().all()) and bool(codes[2, 1, 2].isnan().all())
    assert int(codes.isnan().sum()) == 128 and not bool(cache.views()["v_codes"].float().isnan().any())


def test_random_shapes(B):
    import random
    rng = random.Random(11)
    for i in range(12):
        batch, page = rng.randint(1, 5), rng.choice((16, 32, 64, 128))
        lens, news = [rng.randint(0, 300) for _ in range(batch)], [rng.randint(0, 260) for _ in range(batch)]
        _run(B, lens, news, rng.choice((1, 3, 8)), rng.choice((64, 128)), page, rng.choice((0, 16, 32, 64)), rng.random() < 0.5,
             grid=rng.random() < 0.5, seed=100 + i, n=max(max(news), 1))


def test_faults_of_the_lists_are_reported_and_nothing_else_is_touched(B):
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = _kv(1, 1, 40, 64, g)
    cos, sin = P.rope_tables(30, 64)
    for table, lengths, n_new, rope, code in [([[0, 9]], [0], [40], {}, B.KVQ_PAGED_BAD_PAGE), ([[0, -1]], [0], [40], {}, B.KVQ_PAGED_BAD_PAGE),
                                              ([[0, 1]], [30], [40], {}, B.KVQ_PAGED_BAD_LENGTH), ([[0, 1]], [-3], [10], {}, B.KVQ_PAGED_BAD_LENGTH),
                                              ([[0, 1]], [0], [40], dict(cos=cos, sin=sin), B.KVQ_PAGED_BAD_POSITION),
                                              ([[0, 1]], [2 ** 31 - 1], [40], {}, B.KVQ_PAGED_BAD_LENGTH)]:
        cache = B.PagedCache(3, 1, 64, 32)
        for b in cache.buffers:
            b.fill_(0x55)
        status = P.ints([0])
        B.kvq_paged_append(cache, k, v, P.ints(table), P.ints(lengths), n_new=P.ints(n_new), status_word=status, **rope)
        assert int(status) == code
        assert all(bool((b.view(3, -1)[2] == 0x55).all()) for b in cache.buffers)      # the page that no table names


def test_offsets_beyond_32_bits(B):
    pages = 300_000                                                                    # 128 * 128 * 300 000 = 4.9e9 bytes of codes, twice
    cache = B.PagedCache(pages, 1, 128, 128)
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = _kv(1, 1, 200, 128, g)
    table = P.ints([[pages - 1, pages - 2]])
    B.kvq_paged_append(cache, k, v, table, P.ints([0]))
    small = B.PagedCache(2, 1, 128, 128)
    B.kvq_paged_append(small, k, v, P.ints([[1, 0]]), P.ints([0]))
    for x, y in zip(cache.buffers, small.buffers):
        assert torch.equal(x[-y.numel():], y)
        assert int(x[:-y.numel()].max()) == 0


def test_other_streams_and_graphs(B):
    g = torch.Generator(device="cuda").manual_seed(7)
    k, v = _kv(1, 2, 33, 128, g)
    table, zero = P.ints([[0, 1, 2]]), P.ints([0])
    want, got = B.PagedCache(3, 2, 128, 16), B.PagedCache(3, 2, 128, 16)
    B.kvq_paged_append(want, k, v, table, zero)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        B.kvq_paged_append(got, k, v, table, zero)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want.buffers, got.buffers))
    graph, again = torch.cuda.CUDAGraph(), B.PagedCache(3, 2, 128, 16)
    with torch.cuda.graph(graph):
        B.kvq_paged_append(again, k, v, table, zero)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want.buffers, again.buffers))
