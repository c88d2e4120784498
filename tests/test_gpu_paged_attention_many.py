"""kvq_paged_attn of few rows over many units: short tables, which have a CTA each, and longer ones, which are cut; odd and even numbers of tiles, since two
groups of warps take every other one."""
import random

import pytest
import torch

from tests import paged_testlib as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2605_26266_b200 import binding
    return binding


def _run(B, lens, news, q_heads, kv_heads, d, page, seed, scales=None, **kw):
    gen = torch.Generator().manual_seed(seed)
    cache, table = P.filled(B, lens, news, kv_heads, d, page, gen)
    q = torch.randn(len(lens), q_heads, max(news), d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()
    if scales is not None:
        q *= scales[:, None, None, None].bfloat16()
    lse, status = torch.full(q.shape[:3], 7.0, device="cuda"), P.ints([0])
    out = B.kvq_paged_attn(cache, q, table, P.ints(lens), d ** -0.5, n_new=P.ints(news), lse=lse, status_word=status, **kw)
    want, want_lse = P.attention(cache, q, table, P.ints(lens), d ** -0.5, P.ints(news), **kw)
    P.assert_close(out, want, lse, want_lse, f"{lens} {news} {q_heads}/{kv_heads} d{d} page {page} {kw}")
    assert int(status) == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,n", [(1, 1), (4, 2), (3, 5), (8, 4), (2, 16)])
@pytest.mark.parametrize("batch", [20, 50])                            # 80 and 200 units of four key heads
def test_units_whole_and_cut(B, d, group, n, batch):
    rng = random.Random(100 * group + n + batch)
    lens = [rng.choice((0, 1, 127, 128, 129, 255, 256, 383, rng.randint(0, 2500))) for _ in range(batch)]
    news = [rng.randint(0, n) for _ in range(batch)]
    news[3] = n
    _run(B, lens, news, 4 * group, 4, d, 64, seed=batch + n)


@pytest.mark.parametrize("n", [1, 8, 32])
@pytest.mark.parametrize("window", [0, 200])
def test_units_of_one_to_eight_tiles(B, n, window):
    """Also units that only one of the groups has a tile of, in the middle of others."""
    _run(B, [128 * t - n for t in (1, 2, 3, 4, 5, 6, 7, 8, 1, 1, 2, 1) for _ in range(4)], [n] * 48, 2, 2, 128, 32, seed=n, window=window)


@pytest.mark.parametrize("n", [1, 8, 32])
def test_maxima_that_differ_between_the_groups(B, n):
    """Scores of a hundred and more, so that a tile's weights are nothing beside another's."""
    _run(B, [300, 511, 640, 1000, 4000], [n] * 5, 4, 4, 64, 16, seed=n, scales=torch.tensor([1.0, 20.0, 40.0, 0.0, 60.0], device="cuda"))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("group,longest", [(1, 300), (4, 90), (3, 200)])
def test_chunks_of_one_and_two_query_tiles_in_turn(B, d, causal, group, longest):
    """Many units for each CTA: with one query tile or two, of one key tile or several, in any order; with a window (which causal calls alone have) too."""
    rng = random.Random(longest)
    lens = [rng.choice((0, 1, 100, 128, 250, 500)) for _ in range(150)]
    news = [rng.choice((0, 1, 20, 128 // group, 128 // group + 1, 256 // group, longest)) for _ in range(150)]
    news[0] = longest
    _run(B, lens, news, 4 * group, 4, d, 32, seed=longest + d, causal=causal, window=300 if causal and group == 3 else 0)
