"""kvq_paged_append of so many blocks that CTAs take runs of them: the same, bit for bit, as one call for each sequence."""
import pytest
import torch

from tests import paged_testlib as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2605_26266_b200 import binding
    return binding


LENS = [0, 5, 100, 16, 333, 0, 127, 128, 900, 1, 64, 40]
NEWS = [700, 0, 1, 650, 33, 0, 129, 700, 512, 16, 0, 699]


def _inputs(B, d, page, news, heads=24, seed=0):
    gen, g = torch.Generator().manual_seed(seed), torch.Generator(device="cuda").manual_seed(seed)
    cache, table = P.filled(B, LENS, news, heads, d, page, gen)
    k, v = (torch.randn(len(LENS), heads, 700, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    k[..., 7] *= 30.0
    for x, (b, h, t, c) in ((k, (0, 3, 17, 2)), (v, (3, 0, 649, 5)), (v, (7, 23, 300, 1))):
        x[b, h, t, c] = float("nan")
    k[8, 5, 100, 0], v[11, 9, 3, 3] = float("inf"), -float("inf")
    cos, sin = P.rope_tables(1700, 64)
    positions = torch.randint(0, 1700, (len(LENS), 700), device="cuda", generator=g, dtype=torch.int32)
    return cache, table, k, v, dict(cos=cos, sin=sin, positions=positions)


def _copy(B, cache, heads, d, page):
    return B.PagedCache(cache.desc.pages, heads, d, page, buffers=[x.clone() for x in cache.buffers])


def _one_by_one(B, cache, k, v, table, news, status=None, **rope):
    for b, n in enumerate(news):
        kw = dict(rope, positions=rope["positions"][b:b + 1]) if rope.get("positions") is not None else rope
        B.kvq_paged_append(cache, k[b:b + 1], v[b:b + 1], table[b:b + 1], P.ints([LENS[b]]), n_new=P.ints([n]), status_word=status, **kw)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_runs_are_what_single_blocks_are(B, d, page, ragged, interleaved):
    news = NEWS if ragged else [700] * len(LENS)
    cache, table, k, v, rope = _inputs(B, d, page, news, seed=page + d)
    other = _copy(B, cache, 24, d, page)
    status = P.ints([0])
    rope["interleaved"] = interleaved
    B.kvq_paged_append(cache, k, v, table, P.ints(LENS), n_new=P.ints(news) if ragged else None, status_word=status, **rope)
    _one_by_one(B, other, k, v, table, news, **rope)
    for a, b in zip(cache.buffers, other.buffers):
        assert torch.equal(a, b)
    assert int(status) == 0


@pytest.mark.parametrize("page", [64, 128])
def test_runs_against_the_definition(B, page):
    cache, table, k, v, rope = _inputs(B, 128, page, NEWS, seed=3)
    ref = P.Reference(cache)
    B.kvq_paged_append(cache, k, v, table, P.ints(LENS), n_new=P.ints(NEWS), **rope)
    ref.append(k, v, table, P.ints(LENS), P.ints(NEWS), **rope)
    ref.assert_same(cache)


@pytest.mark.parametrize("ragged", [False, True])
def test_faults_within_runs(B, ragged):
    """A page that the pool does not have, in the middle of a sequence: its tokens are left out, and all others are written."""
    news = NEWS if ragged else [700] * len(LENS)
    cache, table, k, v, rope = _inputs(B, 128, 64, news, seed=8)
    table[3, 4], table[7, 5] = cache.desc.pages, -1
    other = _copy(B, cache, 24, 128, 64)
    status, ones = P.ints([0]), P.ints([0])
    B.kvq_paged_append(cache, k, v, table, P.ints(LENS), n_new=P.ints(news) if ragged else None, status_word=status, **rope)
    _one_by_one(B, other, k, v, table, news, status=ones, **rope)
    for a, b in zip(cache.buffers, other.buffers):
        assert torch.equal(a, b)
    assert int(status) == int(ones) == B.KVQ_PAGED_BAD_PAGE
    status.zero_()
    rope["positions"][0, 13] = 1700
    B.kvq_paged_append(cache, k, v, table.clamp(0, cache.desc.pages - 1), P.ints(LENS), n_new=P.ints(news) if ragged else None, status_word=status, **rope)
    assert int(status) == B.KVQ_PAGED_BAD_POSITION


def test_nothing_new_at_all(B):
    cache, table, k, v, rope = _inputs(B, 128, 128, [0] * len(LENS), seed=4)
    before = [x.clone() for x in cache.buffers]
    B.kvq_paged_append(cache, k, v, table, P.ints(LENS), n_new=P.ints([0] * len(LENS)), **rope)
    for a, b in zip(cache.buffers, before):
        assert torch.equal(a, b)
