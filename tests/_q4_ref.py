"""Plain float64 statements of the 4-bit cache's format and of the operators on it.  Host only (numpy)."""
import numpy as np

from tests import _decode_ref as ref

LEAST, MOST = 2.0 ** -20, 1.875 * 2.0 ** 11


def token_bytes(d):
    return d + d // 16


def page_bytes(page, d):
    return page // 16 * 17 * d


def scale_of(a):
    """a / 7 to four significant bits, ties to even, in range.  (value, distance from the nearest border relative to a / 7)"""
    f = np.clip(np.asarray(a, dtype=np.float64) / 7, LEAST, MOST)
    m, e = np.frexp(f)                                     # m in [0.5, 1)
    s = np.ldexp(np.round(m * 16) / 16, e)
    return np.clip(s, LEAST, MOST), np.abs(m * 16 - np.floor(m * 16) - 0.5) / (m * 16)


def quantise(x):
    """x [..., d] -> (codes [..., d] 0 .. 15, scales [..., d / 32], distance of each element from the nearest border in steps)."""
    x = np.asarray(x, dtype=np.float64)
    g = np.where(np.isnan(x), 0, x).reshape(*x.shape[:-1], -1, 32)
    s, near = scale_of(np.minimum(np.abs(g), 1e300).max(-1))
    t = np.clip(g / s[..., None], -7, 7)
    c = np.round(t)
    border = np.minimum(np.abs(t - np.floor(t) - 0.5), near[..., None] * 100)
    return (c + 8).astype(np.int64).reshape(x.shape), s, border.reshape(x.shape)


def scale_byte(s):
    m, e = np.frexp(s)
    return ((e + 19) * 8 + np.round(m * 16).astype(np.int64) - 8).astype(np.int64)


def byte_scale(b):
    b = np.asarray(b).astype(np.int64)
    return (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 20)


def values(codes, scales):
    return (codes - 8) * np.repeat(scales, 32, -1)


def places(i, d):
    """Where token i of a block has element e's code ([d] byte, [d] shift), for keys and values, and its scales' bytes."""
    e = np.arange(d)
    word, in_word = e // 8, e % 8
    shift = in_word // 2 * 4 + in_word % 2 * 16
    g = np.arange(d // 32)
    row = [0, 4, 1, 5, 2, 6, 3, 7][i % 8] + i // 8 * 8
    k = i * (d // 2) + word * 4 + shift // 8
    v = 8 * d + word // 8 * 512 + row * 32 + word % 8 * 4 + shift // 8
    ks = 16 * d + i % 8 * (d // 16) + g * 2 + i // 8
    vs = 16 * d + d // 2 + g * 16 + i % 8 // 2 * 4 + [0, 2][i % 2] + i // 8
    return k, v, ks, vs, shift % 8


def put(cache, page_id, head, off, d, k, v):
    """Stores (codes, scales) of a token's key and value in cache [pages, heads, bytes] (uint8)."""
    block = cache[page_id, head, off // 16 * 17 * d:][:17 * d]
    pk, pv, ks, vs, shift = places(off % 16, d)
    for (codes, scales), at, s_at in ((k, pk, ks), (v, pv, vs)):
        block[at] = 0
        np.bitwise_or.at(block, at, (codes << shift).astype(np.uint8))
        block[s_at] = scale_byte(scales)


def get(cache, page_id, head, off, d):
    """(key, value) of a token, float64."""
    block = cache[page_id, head, off // 16 * 17 * d:][:17 * d]
    pk, pv, ks, vs, shift = places(off % 16, d)
    return tuple(values((block[at] >> shift & 15).astype(np.int64), byte_scale(block[s_at])) for at, s_at in ((pk, ks), (pv, vs)))


def unpack(cache, page, d):
    """All of a cache [pages, heads, bytes] as keys and values [pages, heads, page, d], float64."""
    n, h, _ = cache.shape
    blocks = cache.reshape(n, h, page // 16, 17 * d)
    out = np.zeros((2, n, h, page // 16, 16, d))
    for i in range(16):
        pk, pv, ks, vs, shift = places(i, d)
        for x, at, s_at in ((0, pk, ks), (1, pv, vs)):
            out[x, :, :, :, i] = values((blocks[..., at] >> shift & 15).astype(np.int64), byte_scale(blocks[..., s_at]))
    return out[0].reshape(n, h, page, d), out[1].reshape(n, h, page, d)


def random_cache(rng, pages, heads, page, d, scale=1.0):
    """Codes of all sixteen values, scales that make values of about `scale` (over a factor of 4)."""
    cache = rng.integers(0, 256, (pages, heads, page_bytes(page, d)), dtype=np.uint8)
    blocks = cache.reshape(pages, heads, page // 16, 17 * d)
    byte = scale_byte(scale_of(np.array(scale * 3.0))[0])
    blocks[..., 16 * d:] = np.clip(byte + rng.integers(-8, 8, blocks[..., 16 * d:].shape), 0, 255)
    return cache


__all__ = ["ref"]
