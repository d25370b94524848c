"""The operators of a sequence that is read token by token, as cases that can be timed and compared.

A model of Transformer blocks that scores a sequence as it grows spends its time on few rows: every weight and every key and value is
read once per token.  Its step is made of

  linear      a linear layer of a few rows whose weights are held in 4 bits, with a scale for each group of inputs (`weights_linear`)
  rotary      positions by rotation of queries and keys, two layouts, part of a head, frequencies for long contexts (`rotary`), and
              the gradients for training (`rotary_grad`)
  cache       new keys and values put into a cache of pages in 8 bits, a scale for each page and head (`cache_append`), and the
              cache read back (`cache_restore`)
  token       attention of one or a few new tokens over that cache (`cache_attention`)
  chunk       the same call for many new tokens

A case is a dict of plain values; `prepare` makes what a serving or training program holds before the call; `run` is one pass, through
the framework's entry points where `own` is true, in elementary binary32 operations otherwise (angles in binary64).

How weights and caches lie (both sides read it):
  weights  codes int32 [n_out / 16][dim / 128][4][16][4] (rounded up): the word (g, row, j) of a block holds the weights of columns
           32 j + 8 g + i, i = 0 .. 7, of that row, four bits each from bit 4 (i / 2) + 16 (i % 2) on; a weight is (code - 8) scale.
           scales bfloat16 [n_out / 16][dim / 128][4][128 / group][4]: of group u and row 4 a + r of a block at (a, u, r)
  caches   codes uint8 (e4m3), keys [pages][kv_heads][head_dim / 16][page_tokens][16], the last of them 16 neighbouring columns, values
           [pages][kv_heads][page_tokens / 16][head_dim][16], the last of them 16 neighbouring tokens; a value is code 2^(exp - 127),
           exps uint8 [pages][kv_heads]; pages int32 [batch][pages of a sequence]
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
TOP = 448.0   # the largest value of e4m3


def _rot(name, op, dtype, batch, tokens, q_heads, kv_heads, head_dim, rotary_dim, interleaved, scaling, far, ragged):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rotary_dim": rotary_dim, "interleaved": interleaved, "scaling": scaling, "far": far, "ragged": ragged}


def _cache(name, dtype, batch, tokens, before, kv_heads, head_dim, page_tokens):
    return {"name": name, "op": "cache", "dtype": dtype, "batch": batch, "tokens": tokens, "before": before, "kv_heads": kv_heads, "head_dim": head_dim,
            "page_tokens": page_tokens}


def _att(name, op, dtype, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, page_tokens, ragged, sides, max_distance):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "q_tokens": q_tokens, "k_tokens": k_tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page_tokens": page_tokens, "ragged": ragged, "sides": sides, "max_distance": max_distance}


def _linear(name, dtype, rows, n_out, dim, group, bias):
    return {"name": name, "op": "linear", "dtype": dtype, "rows": rows, "n_out": n_out, "dim": dim, "group": group, "bias": bias}


def listed():
    return [
        # one new token of one sequence, far into a long context: a few microseconds, the launch counts
        _rot("rotary_token", "rotary", "bf16", 1, 1, 32, 8, 128, 128, False, "parts", 100000, False),
        # a training batch's queries and keys, half layout: bound by memory
        _rot("rotary_train_16k", "rotary", "bf16", 4, 4096, 32, 8, 128, 128, False, "none", 0, False),
        # gradients of a ragged batch in binary32, pairs side by side, part of an odd head
        _rot("rotary_grad_part", "rotary_grad", "f32", 9, 1001, 12, 3, 100, 36, True, "linear", 0, True),
        # one new token of each of many sequences, pages partly full: the last pages are read and written again
        _cache("cache_tokens_64", "bf16", 64, 1, 190, 8, 128, 64),
        # a long prompt put away and brought back, odd lengths: bound by memory
        _cache("cache_prompt_8k", "f16", 2, 8191, 37, 8, 128, 32),
        # one new token against one short cache: latency
        _att("token_short", "token", "f16", 1, 1, 300, 8, 8, 64, 64, False, 1, 64),
        # one new token for each of many long caches of different lengths: bound by reading the caches
        _att("token_long_batch", "token", "bf16", 32, 1, 32768, 32, 8, 128, 64, True, 0, 1),
        # a handful of guessed tokens checked at once, ragged, a head width that fills no tile, small pages, a learned bias
        _att("tokens_checked_5", "token", "f16", 16, 5, 5003, 16, 4, 80, 16, True, 1, 128),
        # a prompt's next part against what is there: bound by the matrix cores
        _att("chunk_2k", "chunk", "bf16", 1, 2048, 16384, 32, 8, 128, 128, False, 0, 1),
        # a small model's layer for one token, odd sizes: latency
        _linear("linear_token_small", "bf16", 1, 1603, 1100, 32, True),
        # a wide model's layer for one token: bound by reading the weights
        _linear("linear_token_wide", "bf16", 1, 32768, 8192, 128, False),
        # a dozen sequences' tokens at once
        _linear("linear_rows_12", "f16", 12, 16384, 4096, 64, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(float(lo) * (float(hi) / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["rotary"] * 2 + ["rotary_grad"] * 2 + ["cache"] * 3 + ["token"] * 4 + ["chunk"] * 2 + ["linear"] * 4)
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    q_heads = kv_heads * rng.choice([1, 1, 2, 4, 7])
    if op in ("rotary", "rotary_grad"):
        head_dim = rng.choice([32, 64, 80, 96, 100, 128, 128, 256])
        rotary_dim = head_dim if rng.random() < 0.6 else max(2, 2 * (_log_int(rng, 4, head_dim) // 2))
        tokens = _log_int(rng, 1, 8000)
        most = (1 << 26) // (tokens * (q_heads + kv_heads) * head_dim)
        c = _rot("", op, rng.choice(["bf16", "f16", "f32"]), max(1, min(most, _log_int(rng, 1, 64))), tokens, q_heads, kv_heads, head_dim, rotary_dim, rng.random() < 0.5,
                 rng.choice(["none", "linear", "parts"]), rng.choice([0, 0, 4000, 300000]), rng.random() < 0.4)
    elif op == "cache":
        head_dim = rng.choice([32, 64, 80, 128, 128])
        tokens, before = rng.choice([1, 1, 1, _log_int(rng, 2, 9), _log_int(rng, 10, 8000)]), rng.choice([0, _log_int(rng, 1, 400)])
        most = (1 << 25) // ((tokens + before) * kv_heads * head_dim)
        c = _cache("", rng.choice(["bf16", "f16"]), max(1, min(most, _log_int(rng, 1, 100))), tokens, before, kv_heads, head_dim, rng.choice([16, 32, 64, 128]))
    elif op in ("token", "chunk"):
        head_dim, page_tokens = rng.choice([32, 64, 80, 128, 128]), rng.choice([16, 32, 64, 64, 128])
        sides, max_distance = rng.choice([0, 0, 1]), rng.choice([8, 40, 128, 500])
        dtype, ragged = rng.choice(["bf16", "f16"]), rng.random() < 0.6
        if op == "token":
            q_tokens, k_tokens = rng.choice([1, 1, 1, 2, 4, 8]), _log_int(rng, 8, 65536)
            batch = max(1, min(_log_int(rng, 1, 64), (1 << 29) // (k_tokens * kv_heads * head_dim)))
        else:
            q_tokens = _log_int(rng, 9, 2000)
            k_tokens = q_tokens + rng.choice([0, _log_int(rng, 1, 12000)])
            each = 100 * 10**9 // (head_dim * 4)   # pairs of a query and a key, over all heads
            while q_tokens * k_tokens * q_heads > each:
                q_tokens, k_tokens = (q_tokens * 3 + 3) // 4, (k_tokens * 3 + 3) // 4
            batch = max(1, min(each // (q_tokens * k_tokens * q_heads), _log_int(rng, 1, 40)))
        c = _att("", op, dtype, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, page_tokens, ragged, sides, max_distance)
    else:
        c = _linear("", rng.choice(["bf16", "f16"]), rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 2, 16), _log_int(rng, 17, 100)]), _log_int(rng, 16, 20000),
                    _log_int(rng, 16, 12000), rng.choice([32, 64, 128]), rng.random() < 0.3)
    del c["name"]
    return c


# ---- what a program holds before the call


def _randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _order(seed, n):
    return np.random.RandomState(int(seed) % (1 << 32)).permutation(n)


def _device(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _frequencies(case):
    """Angle per position of every pair (binary64): 10000^(-2 i / rotary_dim), divided by 8 where positions are to reach eight times as far ("linear"), or only
    where a pair turns less than once over 4096 positions, not where it turns four times, and in between in proportion ("parts")."""
    i = np.arange(case["rotary_dim"] // 2, dtype=np.float64)
    f = 10000.0 ** (-2.0 * i / case["rotary_dim"])
    if case["scaling"] == "linear":
        return f / 8.0
    if case["scaling"] == "parts":
        keep = np.clip((4096.0 * f / (2.0 * np.pi) - 1.0) / 3.0, 0.0, 1.0)
        return f * (keep + (1.0 - keep) / 8.0)
    return f


def _edges(case):
    """Distances at which a new bucket begins: every one up to 16, then about 1.25 apart, the last at max_distance."""
    at, found = 1, []
    while at < case["max_distance"]:
        found.append(at)
        at = at + 1 if at < 16 else max(at + 1, at * 5 // 4)
    return found + [case["max_distance"]]


def _lengths(case):
    """New tokens and all tokens of every sequence, before they are shuffled."""
    n, most, new = case["batch"], case["k_tokens"], case["q_tokens"]
    keys = [min(most, 1 + int(most * (i + 0.5) / n)) for i in range(n)] if case["ragged"] else [most] * n
    return [(min(new, k), k) for k in keys]


def _pages(seed, lengths, page_tokens, columns):
    """Pages of sequences of these lengths, anywhere in the pool, and the pool's size; -1 where a sequence has no page yet."""
    used = [-(-n // page_tokens) for n in lengths]
    total = sum(used) + 3
    order, at = _order(seed + 1, total).astype(np.int32), 0
    pages = np.full((len(lengths), columns), -1, dtype=np.int32)
    for b, n in enumerate(used):
        pages[b, :n] = order[at:at + n]
        at += n
    return pages, total


def _two_to(e):
    """2^e in binary32, e -126 .. 127 (powers and ldexp of torch are off by a rounding here and there)."""
    return ((e.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _exponents(top):
    """The smallest e >= -126 with top <= 448 2^e (448 = 0.875 2^9)."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, e.int() - 9 + (m > 0.875).int(), torch.full_like(e.int(), -126)).clamp(min=-126)


def _lay(x, turned):
    """[pages, heads, place, column] as it lies in a cache."""
    p, h, t, d = x.shape
    return x.view(p, h, t // 16, 16, d).transpose(3, 4).contiguous() if turned else x.view(p, h, t, d // 16, 16).transpose(2, 3).contiguous()


def _fill(gen, pages, heads, page_tokens, head_dim, turned):
    """Codes and exponents of a pool of pages: channels of different sizes, pages of different sizes."""
    codes = torch.empty((pages, heads, page_tokens // 16, head_dim, 16) if turned else (pages, heads, head_dim // 16, page_tokens, 16), dtype=torch.uint8, device="cuda")
    exps = torch.empty((pages, heads), dtype=torch.uint8, device="cuda")
    channel = torch.exp(_randn(gen, heads, 1, head_dim) * 0.7)
    step = max(1, (1 << 27) // (heads * page_tokens * head_dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        x = torch.randn((n, heads, page_tokens, head_dim), generator=gen, device="cuda") * channel * torch.exp(_randn(gen, n, 1, 1, 1) * 0.2)
        e = _exponents(x.abs().amax((2, 3)))
        codes[p:p + step] = _lay((x * _two_to(-e)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8), turned)
        exps[p:p + step] = (e + 127).to(torch.uint8)
    return codes, exps


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt, op = TYPES[case["dtype"]], case["op"]
    s = {"case": case}
    if op in ("rotary", "rotary_grad"):
        b, n, hq, hk, d = (case[k] for k in ("batch", "tokens", "q_heads", "kv_heads", "head_dim"))
        qkv = _randn(gen, b, n, hq + 2 * hk, d, dtype=dt)   # one fused projection's output
        s["q"], s["k"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
        s["freqs"] = _frequencies(case)
        s["amplitude"] = 1.1 if case["scaling"] == "parts" else 1.0
        first = np.random.RandomState(int(seed) % (1 << 32)).randint(case["far"] // 2, case["far"] + 1, size=b)
        if case["ragged"]:   # several sequences packed into each row: positions begin again
            at = np.zeros((b, n), dtype=np.int32)
            for i in range(b):
                cut = 1 + (37 * (i + 3) + int(seed)) % n
                at[i, :cut], at[i, cut:] = first[i] + np.arange(cut), np.arange(n - cut)
            s["positions"], s["q_len"], s["k_len"] = _device(at), None, None
        else:
            s["positions"], s["q_len"] = None, None
            s["k_len"] = _device((first + n).astype(np.int32))
    elif op == "cache":
        b, n, hk, d, t = (case[k] for k in ("batch", "tokens", "kv_heads", "head_dim", "page_tokens"))
        before = np.array([case["before"] * (2 * i + 1) // (2 * b) if b > 1 else case["before"] for i in range(b)])[_order(seed, b)]
        most = case["before"] + n
        columns = -(-most // t)
        pages, total = _pages(seed, (before + n).tolist(), t, columns)
        s["k_codes"], s["k_exps"] = _fill(gen, total, hk, t, d, False)
        s["v_codes"], s["v_exps"] = _fill(gen, total, hk, t, d, True)
        s["pages"], s["tokens"], s["before"] = _device(pages), most, _device(before.astype(np.int32))
        s["k_len"], s["q_len"] = _device((before + n).astype(np.int32)), None
        kv = _randn(gen, b, n, 2 * hk, d)
        kv = (kv * torch.exp(_randn(gen, 2 * hk, d) * 0.7) * torch.exp(_randn(gen, b, n, 1, 1) * 0.3)).to(dt)
        s["k"], s["v"] = kv[:, :, :hk], kv[:, :, hk:]
    elif op in ("token", "chunk"):
        b, lq, lk, hq, hk, d, t = (case[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "head_dim", "page_tokens"))
        lengths = np.array(_lengths(case), dtype=np.int32)[_order(seed, b)]
        pages, total = _pages(seed, lengths[:, 1].tolist(), t, -(-lk // t))
        s["k_codes"], s["k_exps"] = _fill(gen, total, hk, t, d, False)
        s["v_codes"], s["v_exps"] = _fill(gen, total, hk, t, d, True)
        s["pages"], s["q_len"], s["k_len"] = _device(pages), _device(lengths[:, 0]), _device(lengths[:, 1])
        s["q"] = _randn(gen, b, lq, hq + 2 * hk, d, dtype=dt)[:, :, :hq]
        s["edges"] = np.array(_edges(case), dtype=np.int32) if case["sides"] else None
        s["table"] = _randn(gen, len(_edges(case)) + 1, hq, dtype=dt, scale=0.5) if case["sides"] else None
        s["scale"] = 0.5 / math.sqrt(d)
    else:
        rows, n, d, group = (case[k] for k in ("rows", "n_out", "dim", "group"))
        tiles, blocks = -(-n // 16), -(-d // 128)
        u = torch.zeros(tiles * 16, blocks * 128, dtype=torch.uint8, device="cuda") + 8
        u[:n, :d] = (_randn(gen, n, d) * 2.6).round_().clamp_(-8, 7).add_(8).to(torch.uint8)
        u = u.view(tiles, 16, blocks, 4, 4, 4, 2)                                     # [.., row, .., j, g, i / 2, i % 2]
        words = torch.zeros(u.shape[:5], dtype=torch.int32, device="cuda")
        for i in range(4):
            for h in range(2):
                words |= u[..., i, h].int() << (4 * i + 16 * h)
        s["codes"] = words.permute(0, 2, 4, 1, 3).contiguous()                        # [tile, block, g, row, j]
        s["scales"] = (torch.exp(_randn(gen, tiles, blocks, 4, 128 // group, 4) * 0.3) / (2.6 * math.sqrt(d))).to(torch.bfloat16)
        s["x"] = _randn(gen, rows, d, dtype=dt)
        s["bias"] = _randn(gen, n) if case["bias"] else None
    return s


# ---- one pass


def run(s):
    op = s["case"]["op"]
    if own:
        return _OWN[op](s)
    return _PLAIN[op](s)


def _own_rotary(s):
    import paper_2402_02361_amd as P
    return P.rotary(s["q"], s["k"], s["freqs"], positions=s["positions"], q_len=s["q_len"], k_len=s["k_len"], interleaved=s["case"]["interleaved"], amplitude=s["amplitude"])


def _own_rotary_grad(s):
    import paper_2402_02361_amd as P
    return P.rotary_grad(s["q"], s["k"], s["freqs"], positions=s["positions"], q_len=s["q_len"], k_len=s["k_len"], interleaved=s["case"]["interleaved"], amplitude=s["amplitude"])


def _own_cache(s):
    import paper_2402_02361_amd as P
    cache = P.Cache(s["k_codes"], s["v_codes"], s["k_exps"], s["v_exps"], s["pages"])
    P.cache_append(cache, s["k"], s["v"], q_len=s["q_len"], k_len=s["k_len"])
    return P.cache_restore(cache, s["tokens"], s["k_len"], s["k"].dtype)


def _own_token(s):
    import paper_2402_02361_amd as P
    cache = P.Cache(s["k_codes"], s["v_codes"], s["k_exps"], s["v_exps"], s["pages"])
    return P.cache_attention(s["q"], cache, s["table"], s["edges"], q_len=s["q_len"], k_len=s["k_len"], causal=True, scale=s["scale"])


def _own_chunk(s):
    import paper_2402_02361_amd as P
    cache = P.Cache(s["k_codes"], s["v_codes"], s["k_exps"], s["v_exps"], s["pages"])
    return P.cache_attention(s["q"], cache, s["table"], s["edges"], q_len=s["q_len"], k_len=s["k_len"], causal=True, scale=s["scale"], want_lse=True)


def _own_linear(s):
    import paper_2402_02361_amd as P
    c = s["case"]
    return P.weights_linear(s["x"], P.PackedWeights(s["codes"], s["scales"], c["n_out"], c["dim"], c["group"]), bias=s["bias"])


_OWN = {"rotary": _own_rotary, "rotary_grad": _own_rotary_grad, "cache": _own_cache, "token": _own_token, "chunk": _own_chunk, "linear": _own_linear}


# ---- the plain forms


def _positions(s):
    """[batch, tokens], of every token."""
    c = s["case"]
    if s["positions"] is not None:
        return s["positions"].long()
    return (s["k_len"].long() - c["tokens"])[:, None] + torch.arange(c["tokens"], device="cuda")


def _plain_turn(s, back):
    c = s["case"]
    r = c["rotary_dim"]
    angle = _positions(s).double()[..., None] * torch.from_numpy(s["freqs"]).cuda()
    cos, sin = ((f(angle) * s["amplitude"]).float()[:, :, None] for f in (torch.cos, torch.sin))
    if back:
        sin = -sin
    out = []
    for x in (s["q"], s["k"]):
        t = x.float()
        y = t.clone()
        a, b = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        y[..., a] = t[..., a] * cos - t[..., b] * sin
        y[..., b] = t[..., b] * cos + t[..., a] * sin
        out.append(y.to(x.dtype))
    return tuple(out)


def _plain_cache(s):
    """Pages that get tokens, one column of the page table after the other: the exponent is the larger of what the page's tokens have and what the new ones need,
    and older tokens are rounded to it once more."""
    c = s["case"]
    n, t = c["tokens"], c["page_tokens"]
    before, pages = s["before"].long(), s["pages"].long()
    at = before[:, None] + torch.arange(n, device="cuda")                             # place of every new token
    page, place = torch.gather(pages, 1, at // t), at % t
    for codes, exps, x, turned in ((s["k_codes"], s["k_exps"], s["k"], False), (s["v_codes"], s["v_exps"], s["v"], True)):
        x = x.float()
        need = _exponents(x.abs().amax(-1))                                           # [batch, tokens, heads]
        # of every page, the largest exponent that its new tokens need
        most = torch.full(exps.shape, -126, dtype=torch.int32, device="cuda")
        most.scatter_reduce_(0, page.reshape(-1, 1).expand(-1, exps.shape[1]), need.reshape(-1, exps.shape[1]), "amax")
        first = torch.gather(pages, 1, (before // t)[:, None])[:, 0]                  # the pages that hold older tokens, if place > 0
        kept = (before % t)[:, None] > torch.arange(t, device="cuda")                 # [batch, place]
        old = codes[first].view(torch.float8_e4m3fn).float()
        was = exps[first].int() - 127
        now = torch.where(kept[:, :1], torch.maximum(most[first], was), most[first])
        again = (old * _two_to(was - now)[..., None, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        where = kept.view(-1, 1, t // 16, 1, 16) if turned else kept.view(-1, 1, 1, t, 1)
        codes[first] = torch.where(where, again, codes[first])
        most[first] = now
        exps[page] = (most[page] + 127).to(torch.uint8)
        new = (x * _two_to(-most[page])[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)   # [batch, tokens, heads, dim]
        if turned:
            codes[page, :, place // 16, :, place % 16] = new
        else:
            codes[page, :, :, place] = new.unflatten(-1, (-1, 16))
    return _plain_restore(s)


def _dense(s, codes, exps, turned, b):
    """Sequences' values [.., heads, places, dim] in binary32."""
    of = s["pages"][b].long().clamp(min=0)
    x = codes[of].view(torch.float8_e4m3fn).float() * _two_to(exps[of].int() - 127)[..., None, None, None]
    x = (x.transpose(-1, -2) if turned else x.transpose(-2, -3)).movedim(-4, -5)      # [.., heads, page, unit, 16, column] or [.., heads, page, place, unit, 16]
    return x.reshape(*x.shape[:-4], -1, s["case"]["head_dim"])


def _plain_restore(s):
    out = []
    there = torch.arange(s["tokens"], device="cuda")[None, :] < s["k_len"][:, None]
    for codes, exps, turned in ((s["k_codes"], s["k_exps"], False), (s["v_codes"], s["v_exps"], True)):
        x = _dense(s, codes, exps, turned, slice(None)).transpose(1, 2)[:, :s["tokens"]]
        out.append(torch.where(there[:, :, None, None], x, torch.zeros_like(x)).to(s["k"].dtype))
    return tuple(out)


def _plain_attention(s, want_lse):
    c = s["case"]
    lq, lk, hk, d = c["q_tokens"], c["k_tokens"], c["kv_heads"], c["head_dim"]
    group = c["q_heads"] // hk
    o = torch.empty((c["batch"], lq, c["q_heads"], d), dtype=s["q"].dtype, device="cuda")
    lse = torch.empty((c["batch"], c["q_heads"], lq), device="cuda")
    i, j = torch.arange(lq, device="cuda")[:, None], torch.arange(lk, device="cuda")[None, :]
    for b in range(c["batch"]):
        k = _dense(s, s["k_codes"], s["k_exps"], False, b)[:, :lk].contiguous()
        v = _dense(s, s["v_codes"], s["v_exps"], True, b)[:, :lk].contiguous()
        q = s["q"][b].float().view(lq, hk, group, d).permute(1, 2, 0, 3).reshape(hk, group * lq, d)
        t = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(s["scale"]).view(hk, group, lq, lk)
        r = j - i - (s["k_len"][b] - s["q_len"][b])
        if c["sides"]:
            bucket = torch.bucketize((-r).clamp(min=0), torch.from_numpy(s["edges"]).cuda().long(), right=True)
            t += s["table"].float().t()[:, bucket].view(hk, group, lq, lk)
        t.masked_fill_((r > 0) | (j >= s["k_len"][b]) | (i >= s["q_len"][b]), -math.inf)
        top = t.amax(-1, keepdim=True)
        top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        p = t.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p.div_(torch.where(total > 0, total, torch.ones_like(total)))
        o[b] = torch.matmul(p.view(hk, group * lq, lk), v).view(hk, group, lq, d).permute(2, 0, 1, 3).reshape(lq, c["q_heads"], d).to(o.dtype)
        lse[b] = (total.log() + top).view(c["q_heads"], lq)
    return (o, lse) if want_lse else o


def _plain_linear(s):
    c = s["case"]
    shift = torch.arange(4, device="cuda", dtype=torch.int32)[:, None] * 4 + torch.arange(2, device="cuda", dtype=torch.int32)[None, :] * 16
    u = (s["codes"][..., None, None] >> shift) & 15                                   # [tile, block, g, row, j, i / 2, i % 2]
    tiles, blocks = u.shape[:2]
    w = (u.permute(0, 3, 1, 4, 2, 5, 6).reshape(tiles * 16, blocks * 128) - 8).float()
    scale = s["scales"].float().permute(0, 2, 4, 1, 3).reshape(tiles * 16, -1)        # [row, group]
    w = (w.view(tiles * 16, -1, c["group"]) * scale[..., None]).view(tiles * 16, -1)[:c["n_out"], :c["dim"]]
    y = torch.matmul(s["x"].float(), w.t())
    return (y if s["bias"] is None else y + s["bias"]).to(s["x"].dtype)


_PLAIN = {"rotary": lambda s: _plain_turn(s, False), "rotary_grad": lambda s: _plain_turn(s, True), "cache": _plain_cache, "token": lambda s: _plain_attention(s, False),
          "chunk": lambda s: _plain_attention(s, True), "linear": _plain_linear}


# ---- what a pass cannot do without


def work(case):
    size, op = BYTES[case["dtype"]], case["op"]
    if op in ("rotary", "rotary_grad"):
        n = case["batch"] * case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 2 * n * case["head_dim"] * size + 4 * case["batch"] * (case["tokens"] if case["ragged"] else 1) + 4 * case["rotary_dim"], "flops": 3 * n * case["rotary_dim"]}
    if op == "cache":
        b, n, hk, d, t = (case[k] for k in ("batch", "tokens", "kv_heads", "head_dim", "page_tokens"))
        before = [case["before"] * (2 * i + 1) // (2 * b) if b > 1 else case["before"] for i in range(b)]
        new, kept = b * n * hk * d, sum(x + n for x in before) * hk * d
        # tokens in and codes out; codes in and every row of the cache's values out, keys and values each
        return {"bytes": 2 * (new * (size + 1) + kept + b * (case["before"] + n) * hk * d * size) + 2 * hk * sum(-(-(x + n) // t) for x in before), "flops": 2 * (2 * new + kept)}
    if op in ("token", "chunk"):
        lengths, hq, hk, d = _lengths(case), case["q_heads"], case["kv_heads"], case["head_dim"]
        pairs = sum(ql * (kl - ql + 1) + ql * (ql - 1) // 2 for ql, kl in lengths)
        nk, pages = sum(kl for _, kl in lengths), sum(-(-kl // case["page_tokens"]) for _, kl in lengths)
        table = (len(_edges(case)) + 1) * hq * size if case["sides"] else 0
        rows = case["batch"] * case["q_tokens"] * hq
        return {"bytes": (sum(ql for ql, _ in lengths) * hq + rows) * d * size + 2 * nk * hk * d + pages * (2 * hk + 4) + table + (4 * rows if op == "chunk" else 0),
                "flops": 4 * pairs * hq * d}
    rows, n, d = case["rows"], case["n_out"], case["dim"]
    return {"bytes": n * -(-d // 2) + 2 * n * -(-d // case["group"]) + rows * (n + d) * size + (4 * n if case["bias"] else 0), "flops": 2 * rows * n * d}


# ---- the definitions in 64 bits


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("rotary", "rotary_grad"):
        return tuple(_exact_turn(s, x, -1.0 if op == "rotary_grad" else 1.0) for x in (s["q"], s["k"]))
    if op == "cache":
        return tuple(_exact_cache(s, *of) for of in (("k_codes", "k_exps", "k", False), ("v_codes", "v_exps", "v", True)))
    if op == "token":
        return _exact_attention(s)[0]
    if op == "chunk":
        return _exact_attention(s)
    return _exact_linear(s)


def _exact_turn(s, x, sign):
    """As products of complex numbers."""
    c = s["case"]
    r, at = c["rotary_dim"], s["positions"].double() if s["positions"] is not None else None
    if at is None:
        at = torch.stack([torch.arange(k - c["tokens"], k, device="cuda", dtype=torch.float64) for k in s["k_len"].tolist()])
    turn = torch.polar(torch.full((), s["amplitude"], dtype=torch.float64, device="cuda"), sign * at[:, :, None] * torch.tensor(s["freqs"], device="cuda"))[:, :, None]
    y = x.double().clone(memory_format=torch.contiguous_format)
    pairs = y[..., :r].reshape(*y.shape[:3], r // 2, 2) if c["interleaved"] else y[..., :r].reshape(*y.shape[:3], 2, r // 2).transpose(3, 4)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y[..., :r] = turned.reshape(*y.shape[:3], r) if c["interleaved"] else turned.transpose(3, 4).reshape(*y.shape[:3], r)
    return y


def _power(e):
    """2^e in binary64 for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _value(codes):
    """What e4m3 codes stand for: sign, four bits of exponent (bias 7), three of fraction."""
    u = codes.long()
    e, f = (u >> 3) & 15, (u & 7).double()
    return torch.where(u >= 128, -1.0, 1.0) * torch.where(e == 0, f * 2.0 ** -9, (8 + f) * _power(e - 10))


def _nearest(x):
    """The nearest value of e4m3, ties to the even code."""
    step = _power((torch.frexp(x.abs().clamp(min=2.0 ** -6)).exponent - 1) - 3)
    return torch.round(x / step) * step


def _exact_cache(s, codes, exps, name, turned):
    """Page by page, each with what it held before and what comes."""
    c = s["case"]
    n, t = c["tokens"], c["page_tokens"]
    out = torch.zeros(c["batch"], s["tokens"], c["kv_heads"], c["head_dim"], dtype=torch.float64, device="cuda")
    if c["batch"] * (s["tokens"] // t + 1) > 3000:
        return None
    for b, before in enumerate(s["before"].tolist()):
        for i, page in enumerate(s["pages"][b].tolist()):
            lo, hi = i * t, min((i + 1) * t, before + n)
            if hi <= lo:
                break
            held = _value(s[codes][page]).transpose(2, 3) if turned else _value(s[codes][page]).transpose(1, 2)
            held = held.reshape(c["kv_heads"], t, c["head_dim"])
            e = s[exps][page].double()[:, None, None] - 127
            kept, values = max(0, min(before, hi) - lo), torch.zeros(c["kv_heads"], hi - lo, c["head_dim"], dtype=torch.float64, device="cuda")
            if lo + kept < hi:
                new = s[name][b, lo + kept - before:hi - before].double().transpose(0, 1)
                need = torch.ceil(torch.log2(new.abs().amax((1, 2), keepdim=True) / TOP)).clamp(min=-126)
                e_now = torch.maximum(need, e) if kept else need
                values[:, kept:] = _nearest(new * _power(-e_now)) * _power(e_now)
                values[:, :kept] = _nearest(held[:, :kept] * _power(e - e_now)) * _power(e_now)
            else:
                values = held[:, :kept] * _power(e)
            out[b, lo:hi] = values.transpose(0, 1)
    return out


def _exact_attention(s):
    c = s["case"]
    hq, lq, t = c["q_heads"], c["q_tokens"], c["page_tokens"]
    group = hq // c["kv_heads"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((c["batch"], hq, lq), -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, m) in enumerate(zip(s["q_len"].tolist(), s["k_len"].tolist())):
        of = s["pages"][b, :-(-m // t)].long()
        r = torch.arange(m, device="cuda")[None, :] - (torch.arange(n, device="cuda")[:, None] + m - n)
        for h in range(c["kv_heads"]):
            k = (_value(s["k_codes"][of, h]) * _power(s["k_exps"][of, h].long() - 127)[:, None, None, None]).transpose(1, 2).reshape(-1, c["head_dim"])[:m]
            v = (_value(s["v_codes"][of, h]) * _power(s["v_exps"][of, h].long() - 127)[:, None, None, None]).transpose(2, 3).reshape(-1, c["head_dim"])[:m]
            for g in range(h * group, (h + 1) * group):
                w = s["scale"] * (s["q"][b, :n, g].double() @ k.t())
                if c["sides"]:
                    w = w + s["table"][:, g].double()[torch.from_numpy(np.searchsorted(s["edges"], (-r).clamp(min=0).cpu().numpy(), side="right")).cuda()]
                w = torch.where(r <= 0, w, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
                total = torch.logsumexp(w, -1)
                o[b, :n, g], lse[b, g, :n] = torch.exp(w - total[:, None]) @ v, total
    return o, lse


def _exact_linear(s):
    """Row by row of a tile, group by group."""
    c = s["case"]
    tiles, blocks = s["codes"].shape[:2]
    x = torch.zeros(c["rows"], blocks * 128, dtype=torch.float64, device="cuda")
    x[:, :c["dim"]] = s["x"].double()
    y = torch.zeros(c["rows"], tiles, 16, dtype=torch.float64, device="cuda")
    for j in range(4):
        unit = 32 * j // c["group"]
        for g in range(4):
            for i in range(8):
                weight = ((s["codes"][:, :, g, :, j] >> (4 * (i // 2) + 16 * (i % 2))) & 15).double() - 8      # [tile, block, row]
                weight = weight * s["scales"][:, :, :, unit, :].double().reshape(tiles, blocks, 16)
                y += (x[:, 32 * j + 8 * g + i::128] @ weight.permute(1, 0, 2).reshape(blocks, -1)).view(c["rows"], tiles, 16)
    y = y.view(c["rows"], -1)[:, :c["n_out"]]
    return y if s["bias"] is None else y + s["bias"].double()
