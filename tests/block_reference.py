"""The operators of a trainable Transformer block in 64 bits, written from their definitions (numpy, on the CPU), with bounds on what a correct
evaluation in 16-bit operands and binary32 sums may differ by."""
import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # half a step of the type, relative
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}                # half a step where it no longer is relative
F32 = 2.0 ** -24
EXP = 2e-5   # relative error of a softmax weight: binary32 scores of a few tens (2^-24 x 30 x a few roundings) and exp2


def cpu(t):
    return None if t is None else t.detach().to("cpu", torch.float64).numpy() if t.is_floating_point() else t.cpu().numpy()


def buckets(r, edges, two_sided):
    r = np.asarray(r)
    d = np.abs(r) if two_sided else np.maximum(-r, 0)
    n = (np.asarray(edges, np.int64)[None, :] <= d.reshape(-1, 1)).sum(1).reshape(d.shape)
    return n + (r > 0) * (len(edges) + 1) * bool(two_sided)


def attention(q, k, v, table=None, edges=(), q_len=None, k_len=None, causal=False, scale=None, do=None):
    """o, lse and, with do, (dq, dk, dv, dtable); a dict that also holds the bounds' ingredients."""
    batch, lq, hq, d = q.shape
    lk, hk = k.shape[1], k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    group = hq // hk
    two_sided = table is not None and table.shape[0] == 2 * (len(edges) + 1)
    z = lambda *s: np.zeros(s)  # noqa: E731
    out = {"o": z(*q.shape), "o_abs": z(*q.shape), "v_abs": z(*q.shape), "lse": np.full((batch, hq, lq), -np.inf)}
    if do is not None:
        for n, s in (("dq", q.shape), ("dk", k.shape), ("dv", v.shape), ("dq_abs", q.shape), ("dk_abs", k.shape), ("dv_abs", v.shape), ("dq_tiny", q.shape), ("dk_tiny", k.shape)):
            out[n] = z(*s)
        out["dq_round"], out["dk_round"] = z(*q.shape), z(*k.shape)
        if table is not None:
            out["dtable"], out["dtable_abs"], out["dtable_delta"] = z(*table.shape), z(*table.shape), z(*table.shape)
        out["dq_delta"], out["dk_delta"] = z(*q.shape), z(*k.shape)
    for b in range(batch):
        ql, kl = (lq if q_len is None else int(np.clip(q_len[b], 0, lq))), (lk if k_len is None else int(np.clip(k_len[b], 0, lk)))
        if ql == 0 or kl == 0:
            continue
        r = np.arange(kl)[None, :] - (kl - ql + np.arange(ql))[:, None]
        seen = r <= 0 if causal else np.ones_like(r, bool)
        n = buckets(r, edges, two_sided) if table is not None else None
        for h in range(hq):
            qq, kk, vv = q[b, :ql, h], k[b, :kl, h // group], v[b, :kl, h // group]
            with np.errstate(all="ignore"):
                s = scale * (qq @ kk.T) + (table[n, h] if table is not None else 0.0)
                s = np.where(seen, s, -np.inf)
                top = s.max(1, keepdims=True)
                e = np.exp(s - np.where(np.isinf(top), 0, top))
                total = e.sum(1, keepdims=True)
                p = np.where(total > 0, e / np.where(total > 0, total, 1), 0)
                lse = np.where(total[:, 0] > 0, np.log(np.where(total[:, 0] > 0, total[:, 0], 1)) + top[:, 0], -np.inf)
            out["o"][b, :ql, h], out["o_abs"][b, :ql, h], out["lse"][b, h, :ql] = p @ vv, p @ np.abs(vv), lse
            out["v_abs"][b, :ql, h] = (p > 0).astype(float) @ np.abs(vv)
            if do is None:
                continue
            g = do[b, :ql, h]
            dp = g @ vv.T
            dp_abs = np.abs(g) @ np.abs(vv).T
            delta = (p * dp).sum(1, keepdims=True)
            ds = p * (dp - delta)
            ds_abs = p * (dp_abs + (p * dp_abs).sum(1, keepdims=True))
            slip = p * (np.abs(g) * np.abs(p @ vv)).sum(1, keepdims=True)   # times half a step: what delta from a rounded o is off by
            hk_ = h // group
            out["dq"][b, :ql, h] = scale * ds @ kk
            out["dk"][b, :kl, hk_] += scale * ds.T @ qq
            out["dv"][b, :kl, hk_] += p.T @ g
            out["dv_abs"][b, :kl, hk_] += p.T @ np.abs(g)
            for name, m in (("abs", ds_abs), ("round", np.abs(ds)), ("delta", slip)):
                out["dq_" + name][b, :ql, h] = scale * m @ np.abs(kk)
                out["dk_" + name][b, :kl, hk_] += scale * m.T @ np.abs(qq)
            out["dq_tiny"][b, :ql, h] = scale * seen.astype(float) @ np.abs(kk)
            out["dk_tiny"][b, :kl, hk_] += scale * seen.T.astype(float) @ np.abs(qq)
            if table is not None:
                np.add.at(out["dtable"][:, h], n, ds)
                np.add.at(out["dtable_abs"][:, h], n, ds_abs)
                np.add.at(out["dtable_delta"][:, h], n, slip)
    return out


def attention_bounds(ref, dt):
    """Bounds by output: a rounding of the result, one of every softmax weight (or its gradient), and binary32's."""
    u, tiny = UNIT[dt], TINY[dt]
    b = {"o": 1.01 * u * (np.abs(ref["o"]) + ref["o_abs"]) + EXP * ref["o_abs"] + tiny * (ref["v_abs"] + 1)}
    if "dq" in ref:
        b["dv"] = 1.01 * u * (np.abs(ref["dv"]) + ref["dv_abs"]) + EXP * ref["dv_abs"] + tiny
        for n in ("dq", "dk"):
            b[n] = 1.01 * u * (np.abs(ref[n]) + ref[n + "_round"] + ref[n + "_delta"]) + EXP * ref[n + "_abs"] + tiny * (ref[n + "_tiny"] + 1)
        if "dtable" in ref:
            b["dtable"] = 1.01 * u * (np.abs(ref["dtable"]) + ref["dtable_delta"]) + EXP * ref["dtable_abs"] + tiny
    return b


def pack(x):
    """(codes, exponent bytes) of x (float32 or narrower values as float64 [rows, dim])."""
    rows, dim = x.shape
    groups = -(-dim // 32)
    codes, exps = np.zeros((rows, dim), np.int8), np.zeros((rows, groups), np.uint8)
    for r in range(rows):
        for g in range(groups):
            part = x[r, 32 * g:32 * g + 32]
            if not np.isfinite(part).all():
                exps[r, g] = 255
                continue
            top, e = np.abs(part).max(), -126
            while top > 127.0 * 2.0 ** e:
                e += 1
            exps[r, g], codes[r, 32 * g:32 * g + 32] = e + 127, np.rint(part / 2.0 ** e).astype(np.int8)
    return codes, exps


def restore(codes, exps):
    e = np.repeat(exps.astype(np.int64), 32, axis=1)[:, :codes.shape[1]]
    return np.where(e == 255, np.nan, codes.astype(np.float64) * 2.0 ** (np.where(e == 255, 127, e) - 127.0))


def norm(x, f, w_post, w_pre, gate=None, alpha=1.0, eps=1e-6, center=False, dh=None, dy=None):
    """h, y and, with dy, the gradients; "_abs" entries are sums of the sizes of the terms."""
    def unit(v):
        m = v.mean(1, keepdims=True) if center else 0.0
        r = 1 / np.sqrt(((v - m) ** 2).mean(1, keepdims=True) + eps)
        return (v - m) * r, r

    def back(d, d_abs, z, r):
        mid, mid_abs = (d.mean(1, keepdims=True), d_abs.mean(1, keepdims=True)) if center else (0.0, 0.0)
        return (r * (d - mid - z * (d * z).mean(1, keepdims=True)),
                r * (d_abs + mid_abs + np.abs(z) * (d_abs * np.abs(z)).mean(1, keepdims=True)))

    out = {}
    s = 1.0 if gate is None else 1 / (1 + np.exp(-gate))
    z1, r1 = unit(f) if f is not None else (np.zeros_like(x), None)
    u = z1 * w_post if f is not None else np.zeros_like(x)
    out["h"] = alpha * x + s * u
    out["h_abs"] = np.abs(alpha * x) + np.abs(s * u)
    z2, r2 = unit(out["h"])
    out["y"] = z2 * w_pre
    out["y_abs"] = (out["h_abs"] + out["h_abs"].mean(1, keepdims=True)) * r2 * np.abs(w_pre)
    if dy is None:
        return out
    z2_abs = (out["h_abs"] + out["h_abs"].mean(1, keepdims=True)) * r2
    z1_abs = (np.abs(f) + np.abs(f).mean(1, keepdims=True)) * r1 if f is not None else None
    d, d_abs = back(dy * w_pre, np.abs(dy * w_pre), z2, r2)
    d_abs = d_abs * (1 + z2_abs / np.sqrt((z2 ** 2).mean(1, keepdims=True) + 1e-30))
    d, d_abs = d + (0 if dh is None else dh), d_abs + (0 if dh is None else np.abs(dh))
    out["dx"], out["dx_abs"] = alpha * d, np.abs(alpha) * d_abs
    out["dw_pre"], out["dw_pre_abs"] = (dy * z2).sum(0), (np.abs(dy) * z2_abs).sum(0)
    if f is None:
        return out
    out["dw_post"], out["dw_post_abs"] = (d * s * z1).sum(0), (d_abs * s * z1_abs).sum(0)
    if gate is not None:
        out["dgate"], out["dgate_abs"] = d * u * s * (1 - s), d_abs * z1_abs * np.abs(w_post) * s
    out["df"], out["df_abs"] = back(d * s * w_post, d_abs * s * np.abs(w_post), z1, r1)
    out["df_abs"] = out["df_abs"] * (1 + z1_abs / np.sqrt((z1 ** 2).mean(1, keepdims=True) + 1e-30))
    return out
