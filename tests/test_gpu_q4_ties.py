"""Which code and which scale of two neighbours a value on the border between them gets: ties to even, every element compared.

Values go through a cache as they are, and so do keys without a norm where nothing turns; the float64 statement is exact there,
so that nothing has to be left out near a border, and codes and scale bytes are compared themselves."""
import numpy as np
import pytest
import torch

from tests import _decode_ref as ref
from tests import _q4_ref as q4
from tests.test_gpu_decode import binding, clean, dev, i32  # noqa: F401 (binding is a fixture)
from tests.test_gpu_q4 import same_codes

pytestmark = pytest.mark.gpu


def raw(cache, page, d):
    """Codes [tokens, heads, d] and scale bytes [tokens, heads, d / 32] of all keys and of all values."""
    n, h, _ = cache.shape
    blocks = cache.reshape(n, h, page // 16, 17 * d)
    codes, scales = np.zeros((2, n, h, page // 16, 16, d), dtype=np.int64), np.zeros((2, n, h, page // 16, 16, d // 32), dtype=np.int64)
    for i in range(16):
        pk, pv, ks, vs, shift = q4.places(i, d)
        for x, at, s_at in ((0, pk, ks), (1, pv, vs)):
            codes[x, :, :, :, i] = blocks[..., at] >> shift & 15
            scales[x, :, :, :, i] = blocks[..., s_at]
    flat = lambda y: y.transpose(0, 1, 3, 4, 2, 5).reshape(2, n * page, h, -1)  # noqa: E731
    return flat(codes), flat(scales)


def on_borders(rng, *shape):
    """Groups of 32 whose elements are halves of their scale apart; of every other group the scale itself lies on a border."""
    d = shape[-1]
    g = np.zeros((*shape[:-1], d // 32, 32))
    every = q4.byte_scale(np.arange(256))
    at = rng.integers(0, 255, g.shape[:-1])
    at[rng.random(at.shape) < 0.1] = 0                                          # the smallest scale, and the largest
    top = rng.random(at.shape) < 0.1
    tie = rng.random(at.shape) < 0.5
    largest = np.where(tie, (every[at] + every[at + 1]) / 2 * 7, np.where(top, 7 * q4.MOST, 7 * every[at]))
    s, near = q4.scale_of(largest)
    assert np.all(near[tie] == 0)
    g[:] = rng.integers(-13, 14, g.shape) / 2 * s[..., None]
    where = rng.integers(0, 32, at.shape)
    np.put_along_axis(g, where[..., None], (largest * rng.choice([-1, 1], at.shape))[..., None], -1)
    below = (at == 0) & ~tie & ~top & (rng.random(at.shape) < 0.5)              # and below the smallest: no element of 7 steps
    np.put_along_axis(g, where[..., None], np.where(below[..., None], 0.5 * q4.LEAST, np.take_along_axis(g, where[..., None], -1)), -1)
    x = g.reshape(shape)
    assert np.array_equal(torch.tensor(x).to(torch.bfloat16).double().numpy(), x)
    return x


def away(x):
    """Codes and scale bytes with ties away from zero."""
    half_up = lambda y: np.sign(y) * np.floor(np.abs(y) + 0.5)  # noqa: E731
    g = x.reshape(*x.shape[:-1], -1, 32)
    m, e = np.frexp(np.clip(np.abs(g).max(-1) / 7, q4.LEAST, q4.MOST))
    s = np.clip(np.ldexp(half_up(m * 16) / 16, e), q4.LEAST, q4.MOST)
    return (half_up(np.clip(g / s[..., None], -7, 7)) + 8).reshape(x.shape), q4.scale_byte(s)


@pytest.mark.parametrize("rows", [1, 37, 3000])                                 # few rows, and the streaming form
@pytest.mark.parametrize("d,hkv,n_freq,interleaved,turned", [
    (128, 8, 0, False, False), (64, 3, 0, False, False), (128, 4, 64, False, False), (64, 8, 32, True, False), (128, 2, 24, False, False),
    # some of a head turns, the groups behind do not
    (128, 4, 16, False, True), (128, 3, 8, True, True), (64, 8, 16, True, True), (64, 2, 8, False, True), (128, 2, 32, False, True)])
def test_ties_go_to_the_even_code_and_scale(binding, d, hkv, n_freq, interleaved, turned, rows):  # noqa: F811
    rng = np.random.default_rng(1000 * rows + 10 * d + n_freq)
    page = 32
    x = on_borders(rng, rows, 2 * hkv, d)
    pos = rng.integers(1, 131072, rows) if turned else np.zeros(rows, dtype=np.int64)
    q = torch.ones(rows, 2 * hkv, d, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    k, v = (y.transpose(0, 1) for y in dev(x).split([hkv, hkv], 1))
    cache = torch.zeros(-(-rows // page), hkv, q4.page_bytes(page, d), dtype=torch.uint8, device="cuda")
    ctx = binding.Context()
    ctx.sp_qk_norm_rope_q4(q, k, v, i32(pos), torch.tensor(1e4 ** (-np.arange(n_freq) / max(1, n_freq))), torch.empty_like(q), cache, i32(range(rows)), interleaved=interleaved)
    clean(ctx)
    codes, scales = (y[:, :rows] for y in raw(cache.cpu().numpy(), page, d))
    for which, first in ((0, -(-2 * n_freq // 32) if turned else 0), (1, 0)):   # the first group that holds no turned element
        y = x[:, which * hkv:(which + 1) * hkv, first * 32:]
        want, s, _ = q4.quantise(y)
        assert np.array_equal(scales[which][..., first:], q4.scale_byte(s)) and np.array_equal(codes[which][..., first * 32:], want)
        if rows > 1:                                                           # the other rule would be seen
            other, other_s = away(y)
            assert np.mean(other != want) > 0.05 and np.mean(other_s != q4.scale_byte(s)) > 0.05


@pytest.mark.parametrize("rows", [37, 3000])
@pytest.mark.parametrize("norm", [False, True])
def test_of_turned_keys_next_to_none_is_left_out(binding, norm, rows):  # noqa: F811
    """What the comparison of turned keys leaves out as too near a border to say: none of continuous values, so that it compares all."""
    hkv, d, page = 4, 128, 32
    rng = np.random.default_rng(rows + norm)
    x = ref.bf16_values(rng, rows, 2 + 2 * hkv, d)
    freq, pos = 5e5 ** (-np.arange(64) / 64.0), rng.integers(1, 131072, rows)
    w = [ref.bf16_values(rng, d) for _ in range(2)] if norm else [None] * 2
    q, k, v = (y.transpose(0, 1) for y in dev(x).split([2, hkv, hkv], 1))
    cache = torch.zeros(-(-rows // page), hkv, q4.page_bytes(page, d), dtype=torch.uint8, device="cuda")
    ctx = binding.Context()
    ctx.sp_qk_norm_rope_q4(q, k, v, i32(pos), torch.tensor(freq), torch.empty_like(q), cache, i32(range(rows)), None, None, *[y if y is None else dev(y) for y in w])
    clean(ctx)
    got, _ = (c.transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:rows] for c in q4.unpack(cache.cpu().numpy(), page, d))
    want, _ = ref.norm_rope(x[:, 2:2 + hkv].transpose(1, 0, 2), w[1], 1e-6, freq, False, pos)
    # within 1e-9 steps of a border: 2e-9 of the elements are to be expected, and as many groups times 32 for their scales
    assert same_codes(got, want.transpose(1, 0, 2), 1e-9) < 1e-5
    codes, scales = (y[1, :rows] for y in raw(cache.cpu().numpy(), page, d))
    c, s, _ = q4.quantise(x[:, 2 + hkv:])
    assert np.array_equal(codes, c) and np.array_equal(scales, q4.scale_byte(s))
