"""The operators of a sequence read token by token in 64 bits, written from their definitions (numpy, on the CPU)."""
import numpy as np

from block_reference import F32, TINY, UNIT, cpu  # noqa: F401


# ---- rotary

def rotary(x, freqs, positions, interleaved=False, amplitude=1.0, back=False):
    """x [batch, tokens, heads, head_dim], positions [batch, tokens]; the result, and per element the sum of the sizes of its two terms' factors."""
    pairs = len(freqs)
    t = np.asarray(positions, np.longdouble)[..., None] * np.asarray(freqs, np.longdouble)   # (64 bits: 2^31 positions are off by 2^-33)
    c, s = np.cos(t).astype(np.float64)[:, :, None], np.sin(t).astype(np.float64)[:, :, None]
    s = -s if back else s
    y, size = x.copy(), np.abs(x)
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    y[..., a], y[..., b] = amplitude * (x[..., a] * c - x[..., b] * s), amplitude * (x[..., b] * c + x[..., a] * s)
    size[..., a] = size[..., b] = abs(amplitude) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    size[..., 2 * pairs:] = 0.0
    return y, size


# ---- e4m3 and the cache

def e4m3(codes):
    u = np.asarray(codes).astype(np.int64)
    e, f = (u >> 3) & 15, u & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where((u & 127) == 127, np.nan, np.where(u >= 128, -v, v))


VALUES = e4m3(np.arange(127))   # of the codes 0 .. 126, ascending


def to_e4m3(x):
    """Codes of the nearest values, ties to the even code (|x| <= 448); NaN and infinities have code 127."""
    x = np.asarray(x, np.float64)
    size = np.where(np.isfinite(x), np.abs(x), 0.0)
    above = np.minimum(np.searchsorted(VALUES, size, side="left"), 126)
    below = np.maximum(above - 1, 0)
    d = (VALUES[above] - size) - (size - VALUES[below])
    code = np.where(d < 0, above, np.where(d > 0, below, np.where(above % 2 == 0, above, below)))
    code = np.where(VALUES[above] == size, above, code)
    return np.where(np.isfinite(x), code + 128 * (np.signbit(x)), 127).astype(np.uint8)


def exponent(top):
    """The smallest e >= -126 with top <= 448 2^e."""
    e = -126
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


class Page:
    """One head's keys (or values) of a page, token by token."""

    def __init__(self, codes, byte):
        self.codes, self.byte = codes, int(byte)   # [page_tokens, head_dim]

    def append(self, place, x):
        """x [n, head_dim] becomes the tokens from `place` on."""
        finite = np.abs(x[np.isfinite(x)])
        e = exponent(finite.max() if finite.size else 0.0)
        was = self.byte - 127
        if place > 0:
            e = max(e, was)
            if e > was:
                self.codes[:place] = to_e4m3(e4m3(self.codes[:place]) * 2.0 ** (was - e))
        self.byte = e + 127
        self.codes[place:place + len(x)] = to_e4m3(x * 2.0 ** -e)

    def values(self):
        return e4m3(self.codes) * 2.0 ** (self.byte - 127)


def keys_of(codes):
    """A cache's codes of keys [pages, heads, d / 16, t, 16] as [pages, heads, t, d]."""
    p, h, u, t, _ = codes.shape
    return np.ascontiguousarray(codes.transpose(0, 1, 3, 2, 4)).reshape(p, h, t, 16 * u)


def values_of(codes):
    """A cache's codes of values [pages, heads, t / 16, d, 16] as [pages, heads, t, d]."""
    p, h, u, d, _ = codes.shape
    return np.ascontiguousarray(codes.transpose(0, 1, 2, 4, 3)).reshape(p, h, 16 * u, d)


def append(k_codes, k_exps, table, x, q_len, k_len):
    """In place: [pages, heads, t, d] codes and [pages, heads] bytes of keys (or values) after the call."""
    pages, heads, t, _ = k_codes.shape
    for b in range(x.shape[0]):
        n = int(np.clip(q_len[b], 0, x.shape[1]))
        begin = max(int(k_len[b]), 0) - n
        for i in range(table.shape[1]):
            lo, hi = max(begin, i * t), min(begin + n, (i + 1) * t)
            page = table[b, i]
            if hi <= lo or not 0 <= page < pages:
                continue
            for h in range(heads):
                one = Page(k_codes[page, h], k_exps[page, h])
                one.append(lo - i * t, x[b, lo - begin:hi - begin, h])
                k_exps[page, h] = one.byte


def dense(codes, exps, table, tokens, k_len):
    """Values [batch, tokens, heads, d] and which of them are there [batch, tokens]; others are 0."""
    pages, heads, t, d = codes.shape
    out, there = np.zeros((table.shape[0], tokens, heads, d)), np.zeros((table.shape[0], tokens), bool)
    for b in range(table.shape[0]):
        for at in range(min(tokens, max(0, int(k_len[b])))):
            page = table[b, at // t]
            if 0 <= page < pages:
                out[b, at] = e4m3(codes[page, :, at % t]) * 2.0 ** (exps[page].astype(np.float64) - 127)[:, None]
                there[b, at] = True
    return out, there


# ---- weights in 4 bits

def bf16(x):
    """The nearest bfloat16, ties to even (float64 in and out; finite)."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


def pack_weights(w, group):
    """(codes [n_out, dim] 0..15, scales [n_out, groups]) of float32-representable w."""
    n, d = w.shape
    groups = -(-d // group)
    codes, scales = np.full((n, d), 8, np.int64), np.zeros((n, groups))
    for r in range(n):
        for g in range(groups):
            part = w[r, g * group:(g + 1) * group]
            if not np.isfinite(part).all():
                scales[r, g] = np.nan
                continue
            scales[r, g] = bf16(np.float32(np.abs(part).max()) / np.float32(7))
            if scales[r, g] > 0:
                q = np.rint((part.astype(np.float32) / np.float32(scales[r, g])).astype(np.float64))
                codes[r, g * group:(g + 1) * group] = np.clip(q, -8, 7) + 8
    return codes, scales


def lay_weights(codes, scales, group):
    """As a PackedWeights holds them: int32 words, scales (float64)."""
    n, d = codes.shape
    tiles, blocks = -(-n // 16), -(-d // 128)
    words = np.zeros((tiles, blocks, 4, 16, 4), np.uint32)
    laid = np.zeros((tiles, blocks, 4, 128 // group, 4))
    for r in range(16 * tiles):
        for c in range(128 * blocks):
            code = codes[r, c] if r < n and c < d else 8
            j, g, i = c % 128 // 32, c % 32 // 8, c % 8
            words[r // 16, c // 128, g, r % 16, j] |= np.uint32(int(code) << (4 * (i // 2) + 16 * (i % 2)))
        for u in range(scales.shape[1]):
            if r < n:
                laid[r // 16, u * group // 128, r % 16 // 4, u % (128 // group), r % 4] = scales[r, u]
    return words.view(np.int32), laid
