"""The operators of a trainable Transformer block, as cases that can be timed and compared.

The learned cost model reads sequences (the data-movement blocks of a schedule, in their order).  A block that can be
trained, and that can score sequences as they grow, is made of

  attention   self-attention with a learned relative position bias by buckets (`rel_attention`), its gradients
              (`rel_attention_grad`), and the same call for one or a few new tokens against a cache
  norm        the norm behind one block and the norm before the next with the gate and the residual scale between them
              (`gated_norm`), and the gradients (`gated_norm_grad`)
  checkpoint  activations held in 8 bits for the backward pass (`checkpoint_pack`, `checkpoint_restore`), and a linear
              layer's weight gradient taken from them (`checkpoint_wgrad`)

A case is a dict of plain values; `prepare` makes what a training or serving program holds before the call; `run` is one
pass, through the framework's entry points where `own` is true, in elementary binary32 operations otherwise.
"""
import math

import numpy as np
import torch

own = False

GROUP = 32                      # neighbouring values of a row that share a checkpoint's exponent
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


def _att(name, op, dtype, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, causal, ragged, sides, max_distance):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "q_tokens": q_tokens, "k_tokens": k_tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "causal": causal, "ragged": ragged, "sides": sides, "max_distance": max_distance}


def listed():
    return [
        # the drafted set of one task: candidates of 0 to 8 dataflow blocks, the cost model's width; a few microseconds, launches count
        _att("attention_candidates_8", "attention", "bf16", 2048, 8, 8, 1, 1, 64, False, True, 2, 8),
        # sequences of a few hundred tokens, ragged and odd, looking both ways: an encoder's ordinary batch
        _att("attention_encoder_777", "attention", "f16", 16, 777, 777, 12, 12, 64, False, True, 2, 128),
        # one long sequence, heads that share keys, looking back only: bound by the matrix cores
        _att("attention_causal_8k", "attention", "bf16", 1, 8192, 8192, 16, 4, 128, True, False, 1, 128),
        # the gradients at an ordinary batch of ragged sequences
        _att("attention_grad_ragged_500", "attention_grad", "bf16", 16, 500, 500, 12, 12, 64, False, True, 2, 128),
        # the gradients of a long sequence with shared heads
        _att("attention_grad_causal_5k", "attention_grad", "bf16", 1, 5001, 5001, 16, 4, 128, True, False, 1, 128),
        # one new token against one short cache: latency
        _att("token_short", "token", "f16", 1, 1, 300, 8, 8, 64, True, False, 1, 64),
        # one new token for each of many long caches of different lengths: bound by reading the caches
        _att("token_long_batch", "token", "bf16", 32, 1, 32768, 32, 8, 128, True, True, 1, 128),
        # a few hundred rows at the cost model's width, the next layer's input also as a checkpoint: latency
        {"name": "norm_rows_333", "op": "norm", "dtype": "bf16", "rows": 333, "dim": 256, "kind": "rms", "gate": "rows", "alpha": 1.0, "checkpoint": True},
        # a training batch's rows, an odd width, a gate learned as one vector, mean subtracted
        {"name": "norm_train_16k", "op": "norm", "dtype": "f32", "rows": 16384, "dim": 1100, "kind": "layer", "gate": "vector", "alpha": 0.7, "checkpoint": False},
        # the gradients over a large batch, the block's output coming back from its checkpoint: bound by memory
        {"name": "norm_grad_64k", "op": "norm_grad", "dtype": "bf16", "rows": 65536, "dim": 2048, "kind": "rms", "gate": "rows", "alpha": 1.0, "checkpoint": True},
        # activations of a batch put away in 8 bits and brought back: bound by memory
        {"name": "checkpoint_8k_rows", "op": "checkpoint", "dtype": "f32", "rows": 8191, "dim": 1100},
        # a linear layer's weight gradient from its input's checkpoint: bound by the matrix cores
        {"name": "wgrad_64k_rows", "op": "wgrad", "dtype": "bf16", "rows": 65536, "out": 2048, "dim": 1024},
    ]


def _log_int(rng, lo, hi):
    return int(round(float(lo) * (float(hi) / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["attention"] * 3 + ["attention_grad"] * 3 + ["token"] * 2 + ["norm"] * 2 + ["norm_grad"] * 2 + ["checkpoint", "wgrad", "wgrad"])
    dtype = rng.choice(["bf16", "f16"])
    if op in ("attention", "attention_grad", "token"):
        head_dim = rng.choice([32, 64, 64, 80, 128, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        q_heads = kv_heads * rng.choice([1, 1, 2, 4, 7])
        causal = rng.random() < 0.5
        sides = rng.choice([0, 1, 1]) if causal else rng.choice([0, 1, 2, 2])
        max_distance = rng.choice([8, 40, 128, 128, 500])
        ragged = rng.random() < 0.6
        if op == "token":
            q_tokens, k_tokens = rng.choice([1, 1, 1, 2, 3, 4]), _log_int(rng, 1, 65536)
            batch = max(1, min(_log_int(rng, 1, 64), (1 << 29) // (k_tokens * kv_heads * head_dim)))
            causal = True
        else:
            k_tokens = _log_int(rng, 4, 6000)
            q_tokens = k_tokens if rng.random() < 0.75 else max(1, min(k_tokens, _log_int(rng, 5, 1000)))
            each = min(1 << 29, 250 * 10**9 // (head_dim * (10 if op == "attention_grad" else 4)))   # pairs of a query and a key, over all heads
            while q_tokens * k_tokens * q_heads > each:
                q_tokens, k_tokens = (q_tokens * 3 + 3) // 4, (k_tokens * 3 + 3) // 4
            batch = max(1, min(each // (q_tokens * k_tokens * q_heads), _log_int(rng, 1, 1500)))
        return {k: v for k, v in _att("", op, dtype, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, causal, ragged, sides, max_distance).items() if k != "name"}
    if op in ("norm", "norm_grad"):
        dim = _log_int(rng, 24, 8000)
        if rng.random() < 0.6:
            dim = max(32, dim // 32 * 32)
        dtype = rng.choice(["bf16", "f16", "f32"])
        rows = _log_int(rng, 1, max(1, min(200000, (1 << 25) // dim)))
        return {"op": op, "dtype": dtype, "rows": rows, "dim": dim, "kind": rng.choice(["rms", "layer"]), "gate": rng.choice(["none", "rows", "vector"]),
                "alpha": rng.choice([1.0, 0.7]), "checkpoint": rng.random() < 0.5 and dtype != "f32"}
    if op == "checkpoint":
        dim = _log_int(rng, 5, 8000)
        return {"op": op, "dtype": rng.choice(["bf16", "f16", "f32"]), "rows": _log_int(rng, 1, max(1, (1 << 25) // dim)), "dim": dim}
    return {"op": op, "dtype": dtype, "rows": _log_int(rng, 1, 60000), "out": _log_int(rng, 16, 2000), "dim": _log_int(rng, 16, 1000)}


# ---- what a program holds before the call


def _edges(case):
    """Distances at which a new bucket begins: every one up to 16, then about 1.25 apart, the last at max_distance."""
    at, found = 1, []
    while at < case["max_distance"]:
        found.append(at)
        at = at + 1 if at < 16 else max(at + 1, at * 5 // 4)
    return found + [case["max_distance"]]


def _lengths(case):
    """Valid queries and keys of every sequence, before they are shuffled."""
    n, most = case["batch"], case["k_tokens"]
    low = 1 if case["op"] == "token" else 0
    keys = [min(most, low + int((most + 1 - low) * (i + 0.5) / n)) for i in range(n)] if case["ragged"] else [most] * n
    return [(k if case["q_tokens"] == most else case["q_tokens"], k) for k in keys]


def _randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt, op = TYPES[case["dtype"]], case["op"]
    s = {"case": case}
    if op in ("attention", "attention_grad", "token"):
        b, lq, lk, hq, hk, d = (case[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "head_dim"))
        if lq == lk:   # the three parts of one fused projection's output
            qkv = _randn(gen, b, lq, hq + 2 * hk, d, dtype=dt)
            s["q"], s["k"], s["v"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:]
        else:
            s["q"], s["k"], s["v"] = _randn(gen, b, lq, hq, d, dtype=dt), _randn(gen, b, lk, hk, d, dtype=dt), _randn(gen, b, lk, hk, d, dtype=dt)
        order = np.random.RandomState(int(seed) % (1 << 32)).permutation(b)
        lengths = np.array(_lengths(case), dtype=np.int32)[order]
        s["q_len"], s["k_len"] = torch.from_numpy(lengths[:, 0].copy()).cuda(), torch.from_numpy(lengths[:, 1].copy()).cuda()
        s["edges"] = np.array(_edges(case), dtype=np.int32) if case["sides"] else None
        s["table"] = _randn(gen, case["sides"] * (len(_edges(case)) + 1), hq, dtype=dt, scale=0.5) if case["sides"] else None
        s["scale"] = 1.0 / math.sqrt(d)
        if op == "attention_grad":   # what the forward pass left, and the output's gradient
            s["o"], s["lse"] = _plain_attention(s, True)
            s["do"] = _randn(gen, b, lq, hq, d, dtype=dt)
    elif op in ("norm", "norm_grad"):
        n, d = case["rows"], case["dim"]
        s["x"], s["f"] = _randn(gen, n, d, dtype=dt), _randn(gen, n, d, dtype=dt, scale=2.0)
        s["gate"] = {"none": None, "rows": _randn(gen, n, d, dtype=dt) if case["gate"] == "rows" else None,
                     "vector": _randn(gen, d) if case["gate"] == "vector" else None}[case["gate"]]
        s["w_post"], s["w_pre"] = 1.0 + _randn(gen, d, scale=0.2), 1.0 + _randn(gen, d, scale=0.2)
        if op == "norm_grad":
            s["dh"], s["dy"] = _randn(gen, n, d, dtype=dt), _randn(gen, n, d, dtype=dt)
            if case["checkpoint"]:
                s["f_codes"], s["f_exps"] = _plain_pack(s.pop("f"))
    elif op == "checkpoint":
        # rows of very different sizes, as activations have
        s["x"] = (_randn(gen, case["rows"], case["dim"]) * torch.exp(_randn(gen, case["rows"], 1, scale=2.0))).clamp_(-30000, 30000).to(dt)
    else:
        s["dy"] = _randn(gen, case["rows"], case["out"], dtype=dt)
        s["codes"], s["exps"] = _plain_pack(_randn(gen, case["rows"], case["dim"], dtype=dt))
    return s


# ---- one pass


def run(s):
    op = s["case"]["op"]
    if own:
        return _OWN[op](s)
    return _PLAIN[op](s)


def _own_attention(s):
    import paper_2402_02361_amd as P
    c = s["case"]
    return P.rel_attention(s["q"], s["k"], s["v"], s["table"], s["edges"], q_len=s["q_len"], k_len=s["k_len"], causal=c["causal"], scale=s["scale"], want_lse=True)


def _own_token(s):
    import paper_2402_02361_amd as P
    c = s["case"]
    return P.rel_attention(s["q"], s["k"], s["v"], s["table"], s["edges"], q_len=s["q_len"], k_len=s["k_len"], causal=c["causal"], scale=s["scale"])


def _own_attention_grad(s):
    import paper_2402_02361_amd as P
    c = s["case"]
    return P.rel_attention_grad(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["table"], s["edges"], q_len=s["q_len"], k_len=s["k_len"], causal=c["causal"],
                                scale=s["scale"])


def _own_norm(s):
    import paper_2402_02361_amd as P
    c = s["case"]
    h, y, kept = P.gated_norm(s["x"], s["f"], s["w_post"], s["w_pre"], gate=s["gate"], alpha=c["alpha"], eps=EPS, center=c["kind"] == "layer", checkpoint=c["checkpoint"])
    return (h, y, P.checkpoint_restore(kept, y.dtype)) if c["checkpoint"] else (h, y)


def _own_norm_grad(s):
    import paper_2402_02361_amd as P
    c = s["case"]
    f = P.Checkpoint(s["f_codes"], s["f_exps"]) if c["checkpoint"] else s["f"]
    return P.gated_norm_grad(s["dh"], s["dy"], s["x"], f, s["w_post"], s["w_pre"], gate=s["gate"], alpha=c["alpha"], eps=EPS, center=c["kind"] == "layer")


def _own_checkpoint(s):
    import paper_2402_02361_amd as P
    return P.checkpoint_restore(P.checkpoint_pack(s["x"]), s["x"].dtype)


def _own_wgrad(s):
    import paper_2402_02361_amd as P
    return P.checkpoint_wgrad(s["dy"], P.Checkpoint(s["codes"], s["exps"]))


_OWN = {"attention": _own_attention, "token": _own_token, "attention_grad": _own_attention_grad, "norm": _own_norm, "norm_grad": _own_norm_grad,
        "checkpoint": _own_checkpoint, "wgrad": _own_wgrad}


# ---- the plain forms


def _scores(s):
    """Scaled scores with their bias [B, Hq, Lq, Lk] in binary32, and what is masked."""
    c = s["case"]
    lq, lk, group = c["q_tokens"], c["k_tokens"], c["q_heads"] // c["kv_heads"]
    q = s["q"].float().permute(0, 2, 1, 3).contiguous()
    k = s["k"].float().permute(0, 2, 1, 3).repeat_interleave(group, 1)
    t = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"])
    i, j = torch.arange(lq, device="cuda")[:, None], torch.arange(lk, device="cuda")[None, :]
    first = (s["k_len"] - s["q_len"])[:, None, None].long()
    r = j - i - first                                               # [B, Lq, Lk]
    if c["sides"]:
        distance = r.abs() if c["sides"] == 2 else (-r).clamp(min=0)
        bucket = torch.bucketize(distance, torch.from_numpy(s["edges"]).cuda().long(), right=True)
        if c["sides"] == 2:
            bucket = bucket + (r > 0) * (len(s["edges"]) + 1)
        t += s["table"].float().t()[:, bucket].permute(1, 0, 2, 3)
    masked = (i >= s["q_len"][:, None, None]) | (j >= s["k_len"][:, None, None])
    if c["causal"]:
        masked = masked | (r > 0)
    return t, masked[:, None], r


def _softmax(t, masked):
    t = t.masked_fill_(masked, -math.inf)
    top = t.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = t.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(torch.where(total > 0, total, torch.ones_like(total))), (total.log() + top)[..., 0]


def _plain_attention(s, want_lse):
    c = s["case"]
    p, lse = _softmax(*_scores(s)[:2])
    v = s["v"].float().permute(0, 2, 1, 3).repeat_interleave(c["q_heads"] // c["kv_heads"], 1)
    o = torch.matmul(p, v).permute(0, 2, 1, 3).to(s["q"].dtype).contiguous()
    return (o, lse) if want_lse else o


def _plain_attention_grad(s):
    c = s["case"]
    b, lq, lk, hq, hk, d = (c[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "head_dim"))
    dt, group = s["q"].dtype, hq // hk
    t, masked, r = _scores(s)
    p, _ = _softmax(t, masked)
    q, do = (s[n].float().permute(0, 2, 1, 3).contiguous() for n in ("q", "do"))
    k, v = (s[n].float().permute(0, 2, 1, 3).repeat_interleave(group, 1) for n in ("k", "v"))
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = (dp - (p * dp).sum(-1, keepdim=True)).mul_(p)
    dq = torch.matmul(ds, k) * s["scale"]
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q) * s["scale"]
    shared = lambda x: x.view(b, hk, group, lk, d).sum(2).permute(0, 2, 1, 3).to(dt).contiguous()  # noqa: E731
    out = {"dq": dq.permute(0, 2, 1, 3).to(dt).contiguous(), "dk": shared(dk), "dv": shared(dv)}
    if c["sides"]:
        # sums along the diagonals first: rows one place further to the right each, so that column c holds j + lq - 1 - i = c
        wide = torch.nn.functional.pad(ds.flip(2), (0, lq)).view(b, hq, -1)[:, :, :lq * (lk + lq - 1)].view(b, hq, lq, lk + lq - 1).sum(2)
        r = torch.arange(lk + lq - 1, device="cuda") - (lq - 1) - (s["k_len"] - s["q_len"])[:, None].long()
        distance = r.abs() if c["sides"] == 2 else (-r).clamp(min=0)
        bucket = torch.bucketize(distance, torch.from_numpy(s["edges"]).cuda().long(), right=True)
        if c["sides"] == 2:
            bucket = bucket + (r > 0) * (len(s["edges"]) + 1)
        of = (bucket.flatten()[:, None] == torch.arange(s["table"].shape[0], device="cuda")).float()   # [B diagonals, buckets]
        out["dtable"] = torch.matmul(of.t().contiguous(), wide.permute(0, 2, 1).reshape(-1, hq)).to(dt)
    return out["dq"], out["dk"], out["dv"], out.get("dtable")


def _normed(x, w, center):
    x = x - x.mean(-1, keepdim=True) if center else x
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r, x * r * w


def _plain_norm(s):
    c = s["case"]
    center = c["kind"] == "layer"
    u = _normed(s["f"].float(), s["w_post"], center)[2]
    h = c["alpha"] * s["x"].float() + (u if s["gate"] is None else torch.sigmoid(s["gate"].float()) * u)
    y = _normed(h, s["w_pre"], center)[2].to(s["x"].dtype)
    if not c["checkpoint"]:
        return h.to(s["x"].dtype), y
    return h.to(s["x"].dtype), y, _plain_restore(*_plain_pack(y), y.dtype)


def _norm_back(d, z, r, center):
    return r * (d - (d.mean(-1, keepdim=True) if center else 0) - z * (d * z).mean(-1, keepdim=True))


def _plain_norm_grad(s):
    c = s["case"]
    dt, center = s["x"].dtype, c["kind"] == "layer"
    f = _plain_restore(s["f_codes"], s["f_exps"], torch.float32) if c["checkpoint"] else s["f"].float()
    z1, r1, u = _normed(f, s["w_post"], center)
    sig = None if s["gate"] is None else torch.sigmoid(s["gate"].float())
    h = c["alpha"] * s["x"].float() + (u if sig is None else sig * u)
    z2, r2, _ = _normed(h, s["w_pre"], center)
    dy = s["dy"].float()
    dh = s["dh"].float() + _norm_back(dy * s["w_pre"], z2, r2, center)
    du = dh if sig is None else dh * sig
    dgate = None
    if sig is not None:
        dgate = dh * u * sig * (1 - sig)
        dgate = dgate.sum(0) if c["gate"] == "vector" else dgate.to(dt)
    df = _norm_back(du * s["w_post"], z1, r1, center)
    return (dh * c["alpha"]).to(dt), df.to(dt), dgate, (du * z1).sum(0), (dy * z2).sum(0)


def _plain_pack(x):
    """Codes in [-127, 127] and one power of two per group: the smallest 2^e (e >= -126) with max |x| <= 127 2^e, its byte e + 127; a group with
    an infinity or a NaN has byte 255."""
    n, d = x.shape
    groups = -(-d // GROUP)
    t = torch.nn.functional.pad(x.float(), (0, groups * GROUP - d)).view(n, groups, GROUP)
    top = t.abs().amax(-1)
    bad = ~torch.isfinite(t).all(-1)
    m, e = torch.frexp(torch.where(bad, torch.zeros_like(top), top))          # top = m 2^e, m in [0.5, 1)
    e = torch.where(top > 0, e.int() - 7 + (m > 127.0 / 128.0).int(), torch.full_like(e, -126)).clamp(min=-126)
    codes = torch.ldexp(torch.where(bad[..., None], torch.zeros_like(t), t), -e[..., None]).round()
    return codes.to(torch.int8).view(n, -1)[:, :d].contiguous(), torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)


def _plain_restore(codes, exps, dtype):
    n, d = codes.shape
    e = exps.int().repeat_interleave(GROUP, 1)[:, :d]
    t = torch.ldexp(codes.float(), e - 127)
    return torch.where(e == 255, torch.full_like(t, math.nan), t).to(dtype)


def _plain_checkpoint(s):
    return _plain_restore(*_plain_pack(s["x"]), s["x"].dtype)


def _plain_wgrad(s):
    return torch.matmul(s["dy"].float().t(), _plain_restore(s["codes"], s["exps"], torch.float32))


_PLAIN = {"attention": lambda s: _plain_attention(s, True), "token": lambda s: _plain_attention(s, False), "attention_grad": _plain_attention_grad, "norm": _plain_norm,
          "norm_grad": _plain_norm_grad, "checkpoint": _plain_checkpoint, "wgrad": _plain_wgrad}


# ---- what a pass cannot do without


def work(case):
    size, op = BYTES[case["dtype"]], case["op"]
    if op in ("attention", "attention_grad", "token"):
        lengths, hq, hk, d = _lengths(case), case["q_heads"], case["kv_heads"], case["head_dim"]
        if case["causal"]:
            pairs = 0
            for ql, kl in lengths:   # query i sees kl - ql + i + 1 keys, or none
                n, first = ql, kl - ql + 1
                if first < 1:
                    n, first = max(0, ql + first - 1), 1
                pairs += n * first + n * (n - 1) // 2
        else:
            pairs = sum(ql * kl for ql, kl in lengths)
        nq, nk = sum(ql for ql, _ in lengths), sum(kl for _, kl in lengths)
        table = case["sides"] * (len(_edges(case)) + 1) * hq * size
        padded = case["batch"] * case["q_tokens"] * hq * d * size   # outputs are written for every row
        if op == "attention_grad":
            kv = nk * hk * d * size
            return {"bytes": 3 * nq * hq * d * size + 4 * nq * hq + 2 * kv + padded + 2 * case["batch"] * case["k_tokens"] * hk * d * size + 2 * table,
                    "flops": 10 * pairs * hq * d}
        lse = 4 * case["batch"] * case["q_tokens"] * hq if op == "attention" else 0
        return {"bytes": (nq * hq + 2 * nk * hk) * d * size + padded + lse + table, "flops": 4 * pairs * hq * d}
    n, d = case["rows"], case["dim"]
    packed = n * d + n * -(-d // GROUP)
    if op == "norm":
        streams = 4 + (case["gate"] == "rows") + case["checkpoint"]
        return {"bytes": n * d * size * streams + 4 * d * (2 + (case["gate"] == "vector")) + (2 * packed if case["checkpoint"] else 0), "flops": 14 * n * d}
    if op == "norm_grad":
        streams = 5 + 2 * (case["gate"] == "rows")
        return {"bytes": n * d * size * streams + (packed if case["checkpoint"] else n * d * size) + 4 * d * (4 + 2 * (case["gate"] == "vector")), "flops": 40 * n * d}
    if op == "checkpoint":
        return {"bytes": 2 * n * d * size + 2 * packed, "flops": 4 * n * d}
    return {"bytes": n * case["out"] * size + packed + 4 * case["out"] * d, "flops": 2 * n * case["out"] * d}


# ---- the definitions in 64 bits


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "attention":
        return _exact_attention(s)[:2]
    if op == "token":
        return _exact_attention(s)[0]
    if op == "attention_grad":
        return _exact_attention(s)[2:]
    if op == "norm":
        h, z2, _, _, _, _ = _exact_norm(s, s["f"].double())
        y = z2 * s["w_pre"].double()
        return (h, y, None) if case["checkpoint"] else (h, y)
    if op == "norm_grad":
        return _exact_norm_grad(s)
    if op == "checkpoint":
        return _exact_checkpoint(s["x"].double())
    codes, exps = s["codes"].double(), s["exps"].long()
    value = codes * (2.0 ** (exps - 127).double()).repeat_interleave(GROUP, 1)[:, :codes.shape[1]]
    return s["dy"].double().t().contiguous() @ value


def _exact_attention(s):
    c = s["case"]
    hq, group, lq = c["q_heads"], c["q_heads"] // c["kv_heads"], c["q_tokens"]
    grad = c["op"] == "attention_grad"
    zero = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    o, lse = zero(s["q"]), torch.full((c["batch"], hq, lq), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = (zero(s["q"]), zero(s["k"]), zero(s["v"])) if grad else (None, None, None)
    dtable = zero(s["table"]) if grad and c["sides"] else None
    ql, kl = s["q_len"].tolist(), s["k_len"].tolist()
    for b in range(c["batch"]):
        n, m = ql[b], kl[b]
        if n == 0 or m == 0:
            continue
        r = np.arange(m)[None, :] - (np.arange(n)[:, None] + m - n)
        keep = torch.from_numpy(r <= 0 if c["causal"] else np.ones_like(r, dtype=bool)).cuda()
        bucket = None
        if c["sides"]:
            bucket = np.searchsorted(s["edges"], np.abs(r) if c["sides"] == 2 else np.maximum(-r, 0), side="right") + (r > 0) * (len(s["edges"]) + 1) * (c["sides"] == 2)
            bucket = torch.from_numpy(bucket).cuda()
        for h in range(0, hq, max(1, hq if n * m < (1 << 20) else 1)):
            heads = slice(h, h + max(1, hq if n * m < (1 << 20) else 1))
            of = torch.arange(hq, device="cuda")[heads] // group
            q, k, v = s["q"][b, :n, heads].double().transpose(0, 1), s["k"][b, :m].double()[:, of].transpose(0, 1), s["v"][b, :m].double()[:, of].transpose(0, 1)
            t = s["scale"] * (q @ k.transpose(1, 2))
            if bucket is not None:
                t = t + s["table"].double()[bucket][:, :, heads].permute(2, 0, 1)
            t = torch.where(keep, t, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
            total = torch.logsumexp(t, -1)
            p = torch.where(torch.isinf(total)[..., None], torch.zeros_like(t), torch.exp(t - total[..., None]))
            o[b, :n, heads], lse[b, heads, :n] = (p @ v).transpose(0, 1), total
            if not grad:
                continue
            do = s["do"][b, :n, heads].double().transpose(0, 1)
            dp = do @ v.transpose(1, 2)
            ds = p * (dp - (p * dp).sum(-1, keepdim=True))
            dq[b, :n, heads] = s["scale"] * (ds @ k).transpose(0, 1)
            dk[b, :m].index_add_(1, of, s["scale"] * (ds.transpose(1, 2) @ q).transpose(0, 1))
            dv[b, :m].index_add_(1, of, (p.transpose(1, 2) @ do).transpose(0, 1))
            if dtable is not None:
                for one in range(dtable.shape[0]):
                    dtable[one, heads] += (ds * (bucket == one)).sum((1, 2))
    return o, lse, dq, dk, dv, dtable


def _exact_checkpoint(x):
    n, d = x.shape
    t = torch.cat([x, torch.zeros(n, -d % GROUP, dtype=torch.float64, device="cuda")], 1).reshape(n, -1, GROUP)
    top = t.abs().max(-1, keepdim=True).values
    e = torch.log2(top.clamp(min=1e-40) / 127).ceil()
    e = torch.where(127 * 2.0 ** (e - 1) >= top, e - 1, torch.where(127 * 2.0 ** e < top, e + 1, e)).clamp(min=-126)
    return ((t / 2.0 ** e).round() * 2.0 ** e).reshape(n, -1)[:, :d].contiguous()


def _exact_norm(s, f):
    c = s["case"]

    def unit(v):
        middle = v.mean(1, keepdim=True) if c["kind"] == "layer" else 0.0
        spread = ((v - middle) ** 2).mean(1, keepdim=True)
        return (v - middle) / torch.sqrt(spread + EPS), 1 / torch.sqrt(spread + EPS)

    z1, r1 = unit(f)
    gate = torch.ones((), dtype=torch.float64, device="cuda") if s["gate"] is None else 1 / (1 + torch.exp(-s["gate"].double()))
    h = c["alpha"] * s["x"].double() + gate * z1 * s["w_post"].double()
    z2, r2 = unit(h)
    return h, z2, r2, z1, r1, gate


def _exact_norm_grad(s):
    c = s["case"]
    if c["checkpoint"]:
        f = s["f_codes"].double() * (2.0 ** (s["f_exps"].double() - 127)).repeat_interleave(GROUP, 1)[:, :c["dim"]]
    else:
        f = s["f"].double()
    h, z2, r2, z1, r1, gate = _exact_norm(s, f)
    project = lambda g, z: g - z * (g * z).mean(1, keepdim=True) - (g.mean(1, keepdim=True) if c["kind"] == "layer" else 0)  # noqa: E731
    dy = s["dy"].double()
    dh = s["dh"].double() + r2 * project(dy * s["w_pre"].double(), z2)
    df = r1 * project(dh * gate * s["w_post"].double(), z1)
    dgate = None
    if s["gate"] is not None:
        dgate = dh * z1 * s["w_post"].double() * gate * (1 - gate)
        dgate = dgate.sum(0) if c["gate"] == "vector" else dgate
    return c["alpha"] * dh, df, dgate, (dh * gate * z1).sum(0), (dy * z2).sum(0)
