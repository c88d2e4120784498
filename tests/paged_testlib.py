"""The paged 8-bit cache in 64 bits, written from its definition: token by token, without pages in the arithmetic."""
import math

import torch

REL_L2_TOL = 5e-3      # output of the attention.  Its rounding to BF16 is 2^-9 / sqrt(3) = 1.1e-3 of a number of mean mantissa (1.7e-3 as
                       # measured over normal numbers); a query is held to 2^-9 of each channel at worst, which moves a score by
                       # 2^-9 / sqrt(3) |scale q k|, 1.1e-3 times the scores' size (below 2 here), and a weight by that share: 2.2e-3.
                       # Together 2.8e-3; the bound is not twice that.
MAX_ABS_TOL = 2e-2     # values of unit size: the largest output is some 4, its last place 2^-7 of 2 to 4
LSE_TOL = 2e-2         # a log-sum-exp moves as the largest scores do


def round_e4m3(x):
    """x (float64) rounded to the nearest E4M3 number, ties to even; at most 448; NaN stays."""
    ulp = torch.exp2(torch.frexp(x)[1].double().sub(4).clamp(min=-9))
    r = (x / ulp).round() * ulp
    return torch.where(x.isinf(), x.sign() * 448.0, r.clamp(-448.0, 448.0))


def rotate(x, cos, sin, rows, interleaved):
    """x [heads, tokens, d] float32, one rounding per operation; rows: the tables' row of each token."""
    x = x.float()
    if cos is None:
        return x
    half = cos.shape[1]
    c, s = cos[rows], sin[rows]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * c - b * s, b * c + a * s
    return y


def exponent(y):
    """The smallest e >= -64 with the finite numbers of y at most 448 * 2^e."""
    a = float(torch.where(y.isfinite(), y.abs(), 0.0).max()) if y.numel() else 0.0
    if a == 0.0:
        return -64
    m, x = math.frexp(a)
    return max(x - 9 + (m > 0.875), -64)


class Reference:
    """Codes (as numbers) and exponents of a pool, kept on the host's side of the test."""

    def __init__(self, cache):
        d = cache.desc
        self.d = d
        v = cache.views()
        self.codes = {n: v[n + "_codes"].double().clone() for n in "kv"}
        self.exps = {n: v[n + "_scale"].int() - 127 for n in "kv"}
        self.table = None

    def append(self, k, v, page_table, lengths, n_new=None, cos=None, sin=None, positions=None, interleaved=False):
        page = self.d.page
        for b in range(k.shape[0]):
            start = int(lengths[b])
            m = k.shape[2] if n_new is None else int(n_new[b])
            if m == 0:
                continue
            rows = positions[b, :m].long() if positions is not None else torch.arange(start, start + m, device=k.device)
            ys = {"k": rotate(k[b, :, :m], cos, sin, rows, interleaved), "v": v[b, :, :m].float()}
            bad = (ys["k"].isnan().any(-1) | ys["v"].isnan().any(-1))                       # [heads, m]
            for name, y in ys.items():
                for first in range(start // page, (start + m - 1) // page + 1):
                    lo, hi = max(start, first * page), min(start + m, (first + 1) * page)
                    at = int(page_table[b, first])
                    for h in range(self.d.kv_heads):
                        part = y[h, lo - start:hi - start]
                        e = exponent(part)
                        if lo > first * page:
                            old = int(self.exps[name][at, h])
                            if e > old:
                                n = lo - first * page
                                self.codes[name][at, h, :n] = round_e4m3(self.codes[name][at, h, :n] * 2.0 ** (old - e))
                            e = max(e, old)
                        self.exps[name][at, h] = e
                        coded = round_e4m3(part.double() * 2.0 ** -e)
                        nan = bad[h, lo - start:hi - start, None].expand_as(coded)
                        coded = torch.where(nan, torch.nan, coded) if name == "k" else torch.where(coded.isnan(), 0.0, coded)
                        self.codes[name][at, h, lo - first * page:hi - first * page] = coded

    def assert_same(self, cache):
        v = cache.views()
        for n in "kv":
            got = v[n + "_codes"].double()
            same = (got == self.codes[n]) | (got.isnan() & self.codes[n].isnan())
            assert bool(same.all()), f"{n}: {int((~same).sum())} of {same.numel()} codes differ"
            assert torch.equal(v[n + "_scale"].int() - 127, self.exps[n].int()), f"{n}: scales differ"


def attention(cache, q, page_table, lengths, scale, n_new=None, causal=True, window=0, cos=None, sin=None, positions=None,
              interleaved=False):
    """(out, lse) in float64 of what the cache's buffers hold."""
    d, v = cache.desc, cache.views()
    b, hq, n, hd = q.shape
    group = hq // d.kv_heads
    out = torch.zeros(b, hq, n, hd, dtype=torch.float64, device=q.device)
    lse = torch.full((b, hq, n), -math.inf, dtype=torch.float64, device=q.device)
    for i in range(b):
        start = int(lengths[i])
        m = n if n_new is None else int(n_new[i])
        total = start + m
        if m == 0 or total == 0:
            continue
        rows = positions[i, :m].long() if positions is not None else torch.arange(start, total, device=q.device)
        qr = rotate(q[i, :, :m], cos, sin, rows, interleaved).double()
        ids = page_table[i, :-(-total // d.page)].long()
        k, val = ((v[x + "_codes"][ids].double() * torch.exp2(v[x + "_scale"][ids].double() - 127)[..., None, None])
                  .transpose(0, 1).reshape(d.kv_heads, -1, hd)[:, :total] for x in "kv")
        j, at = torch.arange(total, device=q.device), start + torch.arange(m, device=q.device)[:, None]
        sees = torch.ones(m, total, dtype=torch.bool, device=q.device)
        if causal:
            sees = j <= at
        if window:
            sees = sees & (j > at - window)
        for h in range(hq):
            s = (qr[h] @ k[h // group].T * scale).masked_fill(~sees, -math.inf)
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - torch.where(top == -math.inf, 0.0, top)).masked_fill(~sees, 0.0)
            l = w.sum(-1, keepdim=True)
            out[i, h, :m] = torch.where(l == 0, 0.0, (w @ val[h // group]) / l)
            lse[i, h, :m] = (torch.where(top == -math.inf, 0.0, top) + torch.log(l))[:, 0]
    return out, lse


def assert_close(got, want, lse=None, want_lse=None, what=""):
    assert bool(torch.isfinite(got).all()), what
    diff = (got.double() - want)
    rel, big = float(diff.norm() / want.norm().clamp(min=1e-30)), float(diff.abs().max()) if diff.numel() else 0.0
    size = max(float(want.abs().max()) / 4.0, 1.0) if want.numel() else 1.0
    assert rel <= REL_L2_TOL and big <= MAX_ABS_TOL * size, f"{what}: rel-L2 {rel:.3e}, max-abs {big:.3e}"
    if lse is not None:
        empty = want_lse == -math.inf
        assert torch.equal(lse == -math.inf, empty), what
        err = (lse.double() - want_lse)[~empty].abs()
        assert err.numel() == 0 or float(err.max()) <= LSE_TOL, f"{what}: log-sum-exp {float(err.max()):.3e}"


def make_table(lens, news, page, gen, extra=1, width=None):
    """A shuffled page table of sequences of lens + news tokens; unused entries are numbers that no pool has."""
    need = [-(-(a + n) // page) for a, n in zip(lens, news)]
    width = max(need + [1]) if width is None else width
    pages = sum(need) + extra
    order = torch.randperm(pages, generator=gen)[:sum(need)].to(torch.int32)
    table, at = torch.full((len(lens), width), 0x3FFFFFFF, dtype=torch.int32), 0
    for b, c in enumerate(need):
        table[b, :c] = order[at:at + c]
        at += c
    return table.cuda(), pages


def rope_tables(rows, dim):
    inv = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * inv
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def filled(B, lens, news, kv_heads, head_dim, page, gen, spread=True):
    """A cache whose sequences hold lens + news random tokens (written through the reference's own codes, not the append), with
    slots that no token fills full of large codes."""
    table, pages = make_table(lens, news, page, gen)
    cache = B.PagedCache(pages, kv_heads, head_dim, page)
    g = torch.Generator(device="cuda").manual_seed(int(torch.randint(1 << 30, (1,), generator=gen)))
    for n, codes, scale in (("k", 0, 2), ("v", 1, 3)):
        x = torch.randn(pages, kv_heads, page, head_dim, device="cuda", generator=g)
        e = torch.randint(-9, -6, (pages, kv_heads), device="cuda", generator=g) if spread else torch.full((pages, kv_heads), -8, device="cuda")
        x = (x * torch.exp2(-e.float())[..., None, None]).clamp(-448, 448)
        cache.buffers[codes].copy_(x.to(torch.float8_e4m3fn).view(torch.uint8).flatten())
        cache.buffers[scale].copy_((e + 127).to(torch.uint8).flatten())
    kc, vc = (cache.buffers[i].view(pages, kv_heads, page, head_dim) for i in (0, 1))
    for b, (a, m) in enumerate(zip(lens, news)):
        if (a + m) % page:
            at = int(table[b, (a + m) // page])
            kc[at, :, (a + m) % page:], vc[at, :, (a + m) % page:] = 0x7E, 0xFE       # 448 and -448
    return cache, table
