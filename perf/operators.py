"""The operators of the paged 8-bit cache, as timed cases: the append, which rotates keys by their positions, quantizes
and writes them into pages, and the attention over those pages.

A pool of pages holds E4M3 codes [pages, kv_heads, page, head_dim] of keys and of values, and for each page and head one
scale 2^e (a byte, e + 127).  A sequence is a row of the page table and its length.  Tensors are [batch, heads, tokens,
head_dim] BF16.  Fields of a case:

  kind       "append" (kvq_paged_append) or "attn" (kvq_paged_attn)
  batch, q_heads, kv_heads, head_dim, page
  n          new tokens of a sequence (the queries of an "attn" case, which are in the cache already); where `ragged_n`
             is set, the largest of a batch of different counts
  cached     tokens before those; where `ragged` is set, the largest of a batch of different lengths
  causal     a token sees those up to itself; else all of its sequence
  window     of which only the last `window` (0: all)
  rope       channels that are rotated (0: none), `interleaved`: pairs (0, 1), (2, 3)...; else (0, r/2), (1, r/2 + 1)...
  grid       positions are given: a frame's tokens in an order of their own; else a token's place in its sequence
"""
import math

import torch

own = False

E4M3_MAX = 448.0
E_MIN = -64          # the smallest exponent of a scale


def _case(name, kind, batch, q_heads, kv_heads, head_dim, page, n, cached, causal=True, window=0, rope=0,
          interleaved=False, grid=False, ragged=False, ragged_n=False):
    return dict(name=name, kind=kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page=page, n=n,
                cached=cached, causal=causal, window=window, rope=rope, interleaved=interleaved, grid=grid, ragged=ragged,
                ragged_n=ragged_n)


def listed():
    return [
        # one decoding step of eight requests: the smallest append, where a launch is all there is
        _case("append_token", "append", 8, 32, 8, 128, 64, 1, 1000, rope=128, ragged=True),
        # prompts of different lengths, small heads, a quarter of the channels rotated in neighbouring pairs, small pages
        _case("append_ragged", "append", 16, 16, 4, 64, 16, 700, 333, rope=16, interleaved=True, ragged=True, ragged_n=True),
        # one layer of a video transformer: a chunk of 4680 tokens behind eight others, the first page half full
        _case("append_chunk", "append", 1, 24, 24, 128, 128, 4680, 37440, causal=False, rope=128, grid=True),
        # the smallest attention: one token of a short reply, heads of 64 channels
        _case("token_small", "attn", 1, 8, 2, 64, 16, 1, 300, rope=64),
        # a decoding step of 64 requests of different lengths, four query heads to a key head
        _case("token_batch", "attn", 64, 32, 8, 128, 64, 1, 16384, rope=128, ragged=True),
        # a decoding step of one request over the longest cache
        _case("token_long", "attn", 1, 32, 8, 128, 64, 1, 149760, rope=128),
        # a few new tokens over a prefix, every head with its own keys
        _case("few_tokens", "attn", 1, 32, 32, 128, 128, 16, 16384, rope=128),
        # two prompts into an empty cache
        _case("prompt", "attn", 2, 32, 8, 128, 64, 4096, 0, rope=128),
        # partial prefill: a short chunk over a long prefix
        _case("prefix", "attn", 1, 32, 32, 128, 128, 256, 65536),
        # prompts and replies together, heads of 64 channels, a sliding window
        _case("mixed_window", "attn", 12, 16, 4, 64, 32, 511, 8190, window=2048, rope=64, ragged=True, ragged_n=True),
        # one layer of a video transformer: a chunk sees itself and eight earlier ones; the largest
        _case("video", "attn", 1, 24, 24, 128, 128, 4680, 37440, causal=False, rope=128, grid=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = "append" if rng.random() < 0.3 else "attn"
    head_dim = rng.choice((128, 128, 64))
    kv_heads = rng.choice((1, 2, 4, 8, 24, 32))
    q_heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if g * kv_heads <= 64])
    batch = _log_int(rng, 1, 64)
    n = rng.choice((1, 1, _log_int(rng, 2, 32), _log_int(rng, 32, 4680), _log_int(rng, 32, 4680)))
    cached = rng.choice((0, _log_int(rng, 16, 65536), _log_int(rng, 256, 149760), _log_int(rng, 256, 149760)))
    # a drawn case stays below the largest listed ones: in products, in scores, in tokens of the pool and of the append
    def too_much():
        total = cached + n
        if kind == "append":
            return batch * kv_heads * n * head_dim > 14e6 or batch * kv_heads * total * head_dim > 300e6
        return (4.0 * batch * q_heads * n * total * head_dim > 1.5e12 or batch * q_heads * n * total > 3e9
                or batch * kv_heads * total * head_dim > 600e6)
    while too_much():
        if batch > 1 and rng.random() < 0.4:
            batch = (batch + 1) // 2
        elif cached > 4 * n:
            cached = cached // 2
        elif n > 1:
            n = n // 2 + 1 if n > 2 else 1
            cached = cached // 2
        else:
            batch, cached = max(1, batch // 2), cached // 2
    causal = rng.random() < 0.8
    return dict(kind=kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                page=rng.choice((16, 32, 64, 128)), n=n, cached=cached, causal=causal,
                window=rng.choice((0, 0, _log_int(rng, 64, 16384))) if causal else 0,
                rope=rng.choice((0, head_dim, head_dim, head_dim // 2, 16)), interleaved=rng.random() < 0.4,
                grid=rng.random() < 0.25, ragged=rng.random() < 0.6, ragged_n=rng.random() < 0.4)


# ---- sizes of a case ---------------------------------------------------------------------------


def _share(b, step):
    """A fixed spread of shares in [0.1, 1], the first of them 1."""
    return 1.0 - 0.9 * ((b * step) % 1.0)


def _lengths(case):
    """Tokens before the new ones, and new tokens, of each sequence."""
    lens = [int(case["cached"] * _share(b, 0.618034)) if case["ragged"] else case["cached"] for b in range(case["batch"])]
    news = [max(1, int(case["n"] * _share(b, 0.414214))) if case["ragged_n"] else case["n"] for b in range(case["batch"])]
    return lens, news


def _seen(case, length, new):
    """Pairs of a query and a key that it sees, and the first key that any query of the sequence sees."""
    total, w = length + new, case["window"]
    if not case["causal"]:
        return new * total, 0
    if not w:
        return new * length + new * (new + 1) // 2, 0
    short = max(0, min(new, w - 1 - length))             # queries with fewer than `window` keys up to themselves
    full = new - short
    return full * w + short * length + short * (short + 1) // 2, max(0, length + 1 - w)


def work(case):
    d, kv, hq = case["head_dim"], case["kv_heads"], case["q_heads"]
    lens, news = _lengths(case)
    pages = lambda lo, hi: -(-hi // case["page"]) - lo // case["page"]      # noqa: E731
    if case["kind"] == "append":
        tokens = sum(news)
        scales = sum(pages(a, a + n) for a, n in zip(lens, news)) * kv * 2
        return dict(bytes=tokens * kv * (2 * 2 * d + 2 * d) + scales + tokens * (4 * case["rope"] + 4 * case["grid"]), flops=0)
    moved, flops = 0, 0
    for length, new in zip(lens, news):
        pairs, first = _seen(case, length, new)
        keys = length + new - first
        moved += new * hq * d * 4 + kv * (keys * d * 2 + 2 * pages(first, length + new)) + 4 * pages(first, length + new)
        moved += new * (4 * case["rope"] + 4 * case["grid"])
        flops += 4 * d * hq * pairs
    return dict(bytes=moved, flops=flops)


# ---- inputs ------------------------------------------------------------------------------------


def _keys_values(case, tokens, g):
    """Keys with a few large channels in each head and scales of their own for the heads, values of unit size; FP32."""
    h, d = case["kv_heads"], case["head_dim"]
    k = torch.randn(*tokens, h, d, device="cuda", generator=g)
    large = torch.rand(h, d, device="cuda", generator=g).argsort(-1) < 3
    k *= torch.where(large, 4.0, 1.0) * (0.5 + torch.rand(h, 1, device="cuda", generator=g))
    v = torch.randn(*tokens, h, d, device="cuda", generator=g)
    return k, v


def _exponent(a):
    """The smallest e with a <= 448 * 2^e (448 = 0.875 * 2^9), not below E_MIN."""
    m, x = torch.frexp(a)
    return torch.where(a > 0, x - 9 + (m > 0.875), E_MIN).clamp_(min=E_MIN)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    b, kv, d, page = case["batch"], case["kv_heads"], case["head_dim"], case["page"]
    lens, news = _lengths(case)
    in_cache = lens if case["kind"] == "append" else [x + y for x, y in zip(lens, news)]
    need = [-(-(x + y) // page) for x, y in zip(lens, news)]
    width, used = max(need), sum(need)
    pages = used + 2                                     # one that no sequence has, and a spare one for what is dropped
    order = torch.randperm(pages - 1, generator=g, device="cuda")[:used].to(torch.int32).cpu()
    table, at = torch.full((b, width), -1, dtype=torch.int32), 0
    for i, c in enumerate(need):
        table[i, :c] = order[at:at + c]
        at += c
    table = table.cuda()
    # what earlier steps left: each page's tokens in codes under the page's scale
    state = dict(case=case, page_table=table, lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                 n_new=torch.tensor(news, dtype=torch.int32, device="cuda"))
    held = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    slots = torch.arange(width * page, device="cuda").view(1, width, page) < torch.tensor(in_cache, device="cuda").view(b, 1, 1)
    held.view(-1)[(table.long().clamp(min=0)[:, :, None] * page + torch.arange(page, device="cuda"))[slots]] = True
    for name in ("k", "v"):
        state[name + "_codes"] = torch.empty(pages, kv, page, d, dtype=torch.uint8, device="cuda")
        state[name + "_scale"] = torch.empty(pages, kv, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (kv * page * d))
    for p in range(0, pages, step):
        m = held[p:p + step]
        for name, x in zip("kv", _keys_values(case, tuple(m.shape), g)):
            x = (x * m[:, :, None, None]).transpose(1, 2)
            e = _exponent(x.abs().amax((2, 3)))
            state[name + "_codes"][p:p + step] = torch.ldexp(x, -e[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            state[name + "_scale"][p:p + step] = ((e + 127) * m.any(1)[:, None]).to(torch.uint8)
    if case["kind"] == "append":
        k, v = _keys_values(case, (b, case["n"]), g)
        state["k"], state["v"] = (x.transpose(1, 2).to(torch.bfloat16).contiguous() for x in (k, v))
    else:
        q = torch.randn(b, case["q_heads"], case["n"], d, device="cuda", generator=g)
        q *= 0.5 + torch.rand(case["q_heads"], 1, 1, device="cuda", generator=g)
        state["q"] = q.to(torch.bfloat16)
        state["scale"] = d ** -0.5
    state["cos"] = state["sin"] = state["positions"] = None
    if case["rope"]:
        rows = max(x + y for x, y in zip(lens, news)) + 1
        inv = 10000.0 ** (-torch.arange(0, case["rope"], 2, device="cuda", dtype=torch.float64) / case["rope"])
        angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * inv
        state["cos"], state["sin"] = angle.cos().float(), angle.sin().float()
        if case["grid"]:
            t = torch.arange(case["n"], device="cuda", dtype=torch.int64)
            base = state["lengths"].long()[:, None]
            state["positions"] = ((base + t * 31 % case["n"]) % rows).to(torch.int32)
    return state


# ---- the plain forms ---------------------------------------------------------------------------


def _rotate(x, state):
    """x [batch, heads, n, head_dim] in FP32, rotated by the positions of its tokens."""
    case, r = state["case"], state["case"]["rope"]
    if not r:
        return x
    pos = state["positions"]
    if pos is None:
        pos = state["lengths"][:, None] + torch.arange(x.shape[2], device="cuda")
        pos = pos.clamp(max=state["cos"].shape[0] - 1)           # of tokens that a sequence does not have
    c, s = state["cos"][pos.long()][:, None], state["sin"][pos.long()][:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    lo, hi = a * c - b * s, b * c + a * s
    turned = torch.stack((lo, hi), -1).flatten(-2) if case["interleaved"] else torch.cat((lo, hi), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_append(state):
    case, page = state["case"], state["case"]["page"]
    b, kv, n, d = state["k"].shape
    table, lengths, new = state["page_table"].long(), state["lengths"].long(), state["n_new"].long()
    spare = state["k_scale"].shape[0] - 1
    t = torch.arange(n, device="cuda")
    real = t < new[:, None]
    at = lengths[:, None] + t
    phys = torch.where(real, table.gather(1, (at // page).clamp(max=table.shape[1] - 1)), spare)
    slot = at % page
    first = table.gather(1, (lengths // page).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    first = torch.where((lengths % page > 0) & (new > 0), first, spare)               # pages that hold earlier tokens
    for name in "kv":
        x = state[name].float()
        if name == "k":
            x = _rotate(x, state)
        codes, scale = state[name + "_codes"], state[name + "_scale"]
        top = torch.zeros(scale.shape, device="cuda")
        top.index_reduce_(0, phys.flatten(), x.abs().amax(-1).transpose(1, 2).reshape(b * n, kv), "amax")
        e = _exponent(top)
        old = scale[first].int() - 127
        grown = torch.maximum(old, e[first])
        e[first] = grown
        shift = (old - grown)[:, :, None, None]
        codes[first] = torch.ldexp(codes[first].view(torch.float8_e4m3fn).float(), shift).to(torch.float8_e4m3fn).view(torch.uint8)
        coded = torch.ldexp(x.transpose(1, 2), -e[phys][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        codes[phys.flatten(), :, slot.flatten()] = coded.reshape(b * n, kv, d)
        scale[phys.flatten()] = (e[phys.flatten()] + 127).to(torch.uint8)
    return _cache_of(state)


def _cache_of(state):
    """The pool without its spare page."""
    return {**{x: state[x][:-1].view(torch.float8_e4m3fn) for x in ("k_codes", "v_codes")},
            **{x: state[x][:-1] for x in ("k_scale", "v_scale")}}


def _plain_attn(state):
    case = state["case"]
    b, hq, n, d = state["q"].shape
    kv, table = case["kv_heads"], state["page_table"].long().clamp(min=0)

    def gathered(name):
        codes = state[name + "_codes"][table].view(torch.float8_e4m3fn).float()                # [b, width, kv, page, d]
        x = torch.ldexp(codes, (state[name + "_scale"][table].int() - 127)[..., None, None])
        return x.transpose(1, 2).reshape(b, kv, -1, d)

    q = _rotate(state["q"].float(), state).reshape(b, kv, hq // kv * n, d)
    s = (q @ gathered("k").transpose(-1, -2)).mul_(state["scale"]).view(b, hq, n, -1)
    at = state["lengths"][:, None] + torch.arange(n, device="cuda")                             # [b, n]
    key = torch.arange(s.shape[-1], device="cuda")
    sees = key < (state["lengths"] + state["n_new"])[:, None, None]
    if case["causal"]:
        sees = sees & (key <= at[..., None])
    if case["window"]:
        sees = sees & (key > at[..., None] - case["window"])
    sees = sees & (torch.arange(n, device="cuda") < state["n_new"][:, None])[..., None]
    s.masked_fill_(~sees[:, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = s.sum(-1, keepdim=True)
    v = gathered("v").masked_fill_(~sees.any(1)[:, None, :, None], 0.0)
    o = (s.view(b, kv, -1, s.shape[-1]) @ v).view(b, hq, n, d)
    return torch.where(total > 0, o / total, 0.0).to(torch.bfloat16)


def run(state):
    case = state["case"]
    if not own:
        return _plain_append(state) if case["kind"] == "append" else _plain_attn(state)
    from paper_2605_26266_b200 import binding as kvq
    cache = state.get("cache")
    if cache is None:                                     # the handle of the pool, which a program makes once
        cache = state["cache"] = kvq.PagedCache(state["k_scale"].shape[0], case["kv_heads"], case["head_dim"], case["page"],
                                                buffers=[state[x] for x in ("k_codes", "v_codes", "k_scale", "v_scale")])
    rope = dict(cos=state["cos"], sin=state["sin"], positions=state["positions"], interleaved=case["interleaved"])
    if case["kind"] == "append":
        kvq.kvq_paged_append(cache, state["k"], state["v"], state["page_table"], state["lengths"], n_new=state["n_new"], **rope)
        return _cache_of(state)
    return kvq.kvq_paged_attn(cache, state["q"], state["page_table"], state["lengths"], state["scale"], n_new=state["n_new"],
                              causal=case["causal"], window=case["window"], **rope)


# ---- in 64 bits --------------------------------------------------------------------------------


def _turned(x, state, i):
    """Sequence i's rows x [heads, tokens, head_dim] as complex numbers times e^(i angle), in 64 bits."""
    case, r = state["case"], state["case"]["rope"]
    if not r:
        return x
    m = x.shape[1]
    rows = state["positions"][i, :m].long() if state["positions"] is not None else int(state["lengths"][i]) + torch.arange(m, device="cuda")
    turn = torch.complex(state["cos"][rows].double(), state["sin"][rows].double())
    y = x.clone()
    if case["interleaved"]:
        y[..., :r] = torch.view_as_real(torch.view_as_complex(x[..., :r].unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
    else:
        z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    return y


def _to_e4m3(x):
    """x rounded to the nearest E4M3 number (ties to the even one): steps of 2^(floor(log2 |x|) - 3), and of 2^-9 below 2^-6."""
    ulp = torch.exp2(torch.frexp(x)[1].double().sub_(4).clamp_(min=-9))
    return (x / ulp).round_() * ulp


def _exact_append(state):
    case, page = state["case"], state["case"]["page"]
    res = {}
    for name in "kv":
        codes = state[name + "_codes"].view(torch.float8_e4m3fn).double()
        exps = state[name + "_scale"].double() - 127
        for i in range(case["batch"]):
            start, m = int(state["lengths"][i]), int(state["n_new"][i])
            x = state[name][i, :, :m].double()
            if name == "k":
                x = _turned(x, state, i)
            for p in range(start // page, -(-(start + m) // page)):
                lo, hi = max(start, p * page), min(start + m, (p + 1) * page)
                at, part = int(state["page_table"][i, p]), x[:, lo - start:hi - start]
                top = part.abs().amax((1, 2))
                e = torch.ceil(torch.log2(top / E4M3_MAX))
                e = (e - (top <= E4M3_MAX * torch.exp2(e - 1)).double()).clamp(min=E_MIN)      # a logarithm just above a whole number
                if lo > p * page:
                    was = exps[at].clone()
                    e = torch.maximum(e, was)
                    codes[at] = _to_e4m3(codes[at] * torch.exp2(was - e)[:, None, None])
                exps[at] = e
                codes[at, :, lo - p * page:hi - p * page] = _to_e4m3(part * torch.exp2(-e)[:, None, None])
        res[name + "_codes"], res[name + "_scale"] = codes[:-1], None
    return res


def _exact_attn(state):
    case, page = state["case"], state["case"]["page"]
    b, hq, n, d = state["q"].shape
    group = hq // case["kv_heads"]
    out = torch.zeros(b, hq, n, d, dtype=torch.float64, device="cuda")
    for i in range(b):
        start, m = int(state["lengths"][i]), int(state["n_new"][i])
        total = start + m
        ids = state["page_table"][i, :-(-total // page)].long()
        q = _turned(state["q"][i, :, :m].double(), state, i)
        place, keys = start + torch.arange(m, device="cuda")[:, None], torch.arange(total, device="cuda")
        hidden = torch.zeros(m, total, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= keys > place
        if case["window"]:
            hidden |= keys <= place - case["window"]
        for h in range(case["kv_heads"]):
            k, v = (state[x + "_codes"][ids, h].view(torch.float8_e4m3fn).double()
                    * torch.exp2(state[x + "_scale"][ids, h].double() - 127)[:, None, None] for x in "kv")
            k, v = k.reshape(-1, d)[:total], v.reshape(-1, d)[:total]
            for j in range(h * group, (h + 1) * group):
                s = torch.einsum("md,kd->mk", q[j], k) * state["scale"]
                out[i, j, :m] = torch.softmax(s.masked_fill_(hidden, -math.inf), -1) @ v
    return out


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_append(state) if case["kind"] == "append" else _exact_attn(state)
