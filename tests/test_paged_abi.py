"""The paged cache's entry points reject bad arguments on the host, before they touch a device; no GPU needed."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_26266_b200", "csrc", "paged")


@pytest.fixture(scope="module")
def b():
    from paper_2605_26266_b200 import build
    build.build_library()
    from paper_2605_26266_b200 import binding
    return binding


def cache_of(b, kv_heads=2, head_dim=128, page=64, flags=0, pages=10, ptr=0x10000):
    return b.kvq_paged_cache(kv_heads, head_dim, page, flags, pages, ptr, ptr, ptr, ptr)


def test_sizes(b):
    assert b.kvq_paged_cache_bytes(cache_of(b)) == [10 * 2 * 64 * 128] * 2 + [20] * 2
    out = (C.c_size_t * 4)()
    for bad, want in [(dict(head_dim=96), b.KVQ_ERR_UNSUPPORTED), (dict(page=48), b.KVQ_ERR_UNSUPPORTED), (dict(page=256), b.KVQ_ERR_UNSUPPORTED),
                      (dict(pages=0), b.KVQ_ERR_INVALID_ARG), (dict(kv_heads=0), b.KVQ_ERR_INVALID_ARG), (dict(flags=1), b.KVQ_ERR_INVALID_ARG),
                      (dict(pages=2 ** 31), b.KVQ_ERR_UNSUPPORTED), (dict(kv_heads=70000), b.KVQ_ERR_UNSUPPORTED)]:
        assert b.lib.kvq_paged_cache_bytes(C.byref(cache_of(b, **bad)), out) == want, bad
    assert b.lib.kvq_paged_cache_bytes(None, out) == b.KVQ_ERR_INVALID_ARG
    assert b.lib.kvq_paged_cache_bytes(C.byref(cache_of(b)), None) == b.KVQ_ERR_INVALID_ARG


def calls(b, cache=None, seqs=None, rope=None, x=0x1000, strides=None, n=4, q_heads=4, scale=0.1, window=0, flags=1):
    """Status of an append and of an attention call with these arguments."""
    cache = cache_of(b) if cache is None else cache
    seqs = b.kvq_paged_batch(1, 8, 8, 0x1000, 0x1000, None) if seqs is None else seqs
    s = b.kvq_strides(4 * 128 * 4, 128 * 4, 128) if strides is None else strides
    r = C.byref(rope) if rope is not None else None
    a = b.lib.kvq_paged_append(C.byref(cache), C.byref(seqs), r, x, s, x, s, n, None, None)
    t = b.lib.kvq_paged_attn(C.byref(cache), C.byref(seqs), r, x, s, q_heads, n, x, s, scale, window, flags, None, None, 0, None, None)
    return a, t


def test_refusals(b):
    I, U, A, OK = b.KVQ_ERR_INVALID_ARG, b.KVQ_ERR_UNSUPPORTED, b.KVQ_ERR_ALIGNMENT, b.KVQ_OK
    assert calls(b, n=0) == (OK, OK)
    assert calls(b, seqs=b.kvq_paged_batch(0, 8, 8, None, None, None)) == (OK, OK)
    for want, kw in [(I, dict(cache=cache_of(b, ptr=None))), (A, dict(cache=cache_of(b, ptr=0x10008))), (U, dict(cache=cache_of(b, head_dim=32))),
                     (I, dict(seqs=b.kvq_paged_batch(1, 8, 8, None, 0x1000, None))), (I, dict(seqs=b.kvq_paged_batch(1, 8, 8, 0x1000, None, None))),
                     (I, dict(seqs=b.kvq_paged_batch(-1, 8, 8, 0x1000, 0x1000, None))), (I, dict(seqs=b.kvq_paged_batch(2, 8, 4, 0x1000, 0x1000, None))),
                     (A, dict(seqs=b.kvq_paged_batch(1, 8, 8, 0x1002, 0x1000, None))), (A, dict(seqs=b.kvq_paged_batch(1, 8, 8, 0x1000, 0x1000, 0x1001))),
                     (U, dict(seqs=b.kvq_paged_batch(70000, 8, 8, 0x1000, 0x1000, None))), (U, dict(seqs=b.kvq_paged_batch(1, 2 ** 30, 2 ** 30, 0x1000, 0x1000, None))),
                     (I, dict(x=None)), (A, dict(x=0x1004)), (A, dict(strides=b.kvq_strides(2048, 512, 100))), (I, dict(strides=b.kvq_strides(2048, 512, 0))),
                     (I, dict(strides=b.kvq_strides(2048, -8, 128))), (I, dict(n=-1)),
                     (I, dict(rope=b.kvq_rope(None, 0x1000, None, 0, 9, 64, 0))), (I, dict(rope=b.kvq_rope(0x1000, 0x1000, None, 0, 0, 64, 0))),
                     (I, dict(rope=b.kvq_rope(0x1000, 0x1000, None, 0, 9, 144, 0))), (U, dict(rope=b.kvq_rope(0x1000, 0x1000, None, 0, 9, 40, 0))),
                     (I, dict(rope=b.kvq_rope(0x1000, 0x1000, None, 0, 9, 64, 2))), (A, dict(rope=b.kvq_rope(0x1004, 0x1000, None, 0, 9, 64, 0))),
                     (A, dict(rope=b.kvq_rope(0x1000, 0x1000, 0x1002, 0, 9, 64, 0))), (I, dict(rope=b.kvq_rope(0x1000, 0x1000, None, -1, 9, 64, 0)))]:
        assert calls(b, **kw) == (want, want), kw
    for want, kw in [(I, dict(q_heads=5)), (I, dict(q_heads=0)), (I, dict(scale=0.0)), (I, dict(scale=float("nan"))), (I, dict(scale=1e31)), (I, dict(flags=2)),
                     (I, dict(window=-1)), (I, dict(window=5, flags=0)), (U, dict(q_heads=70000)), (U, dict(n=2 ** 31))]:
        assert calls(b, **kw)[1] == want, kw
    size = C.c_size_t(0)
    seqs = b.kvq_paged_batch(1, 8, 8, None, None, None)                       # sizes are asked for without pointers
    assert b.lib.kvq_paged_attn_workspace_bytes(C.byref(cache_of(b, ptr=None)), C.byref(seqs), 4, 5, 1, C.byref(size)) == OK
    assert b.lib.kvq_paged_attn_workspace_bytes(C.byref(cache_of(b)), C.byref(seqs), 3, 5, 1, C.byref(size)) == I
    assert b.lib.kvq_paged_attn_workspace_bytes(C.byref(cache_of(b)), C.byref(seqs), 4, 5, 1, None) == I


def test_the_binding_takes_no_other_tensors(b):
    import torch
    cache = b.PagedCache(4, 2, 64, 16, device="cpu")
    assert [tuple(v.shape) for v in cache.views().values()] == [(4, 2, 16, 64)] * 2 + [(4, 2)] * 2
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    table, lengths = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for k in (x, x.float(), x[..., :32]):
        with pytest.raises(AssertionError):
            b.kvq_paged_append(cache, k, x, table, lengths)
        with pytest.raises(AssertionError):
            b.kvq_paged_attn(cache, k, table, lengths, 0.1)
    with pytest.raises(AssertionError):
        b.PagedCache(4, 2, 64, 16, buffers=[torch.zeros(3, dtype=torch.uint8)] * 4)


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_every_kernel_may_start_early_and_waits(b):
    """Kernels of a call are launched programmatically: each waits for the grid before it ahead of letting the next one start, and reads
    global memory with ordinary loads."""
    for name in sorted(n for n in os.listdir(CSRC) if n.endswith((".cu", ".cuh"))):
        text = source(name)
        assert "<<<" not in text and "__ldg(" not in text and ".nc." not in text
        for body in text.split("__global__ ")[1:]:
            wait, allow = body.find("wait_for_previous_grid();"), body.find("allow_next_grid();")
            assert 0 <= wait < allow, (name, body[:80])


def test_a_site_code_names_one_wait(b):
    """The codes of the kernels' waits are those that the header lists; faults of the lists are arguments', not time-outs."""
    with open(os.path.join(ROOT, "include", "kvq.h")) as f:
        header = f.read()
    listed = header[header.index("Few rows: 601"):header.index("#define KVQ_PAGED_BAD_PAGE")]
    codes = {int(c) for c in re.findall(r"\b[67]\d\d\b", listed)}
    found = []
    for name in ("attn_few.cu", "attn_chunk.cu"):
        found += [int(c) for c in re.findall(r"cx\.wait\([^;]*?, (\d{3})\)", source(name))]
    assert set(found) == codes
    assert {c for c in found if found.count(c) > 1} <= {711}                  # the keys of a segment's first tile, and of the next ones
    for word in (b.KVQ_PAGED_BAD_PAGE, b.KVQ_PAGED_BAD_POSITION, b.KVQ_PAGED_BAD_LENGTH):
        assert b.kvq_status_word_result(word) == b.KVQ_ERR_INVALID_ARG
    for word in codes:
        assert b.kvq_status_word_result(word) == b.KVQ_ERR_TIMEOUT
