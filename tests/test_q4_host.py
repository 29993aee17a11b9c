"""The calls on a 4-bit cache refuse what they do not support before anything is launched, and the plain statements that the
GPU tests compare with say what they should.  No GPU."""
import ctypes
import struct

import numpy as np
import pytest
import torch

from tests import _q4_ref as q4
from tests.test_decode_host import ADDR, CTX, INV, UNS, view


@pytest.fixture(scope="module")
def lib():
    from paper_2505_19578_b200 import binding, build
    build.build()
    return binding.load()


def cache(pages=10, heads=2, page=16, d=64, s_page=None, s_head=None, data=ADDR):
    """An sp_q4_cache as bytes."""
    n = page // 16 * 17 * d
    return struct.pack("P6q", data, pages, heads, page, d, heads * n if s_page is None else s_page, n if s_head is None else s_head)


BAD_CACHES = [
    (None, INV), (cache(data=0), INV), (cache(data=ADDR + 8), INV), (cache(pages=0), INV), (cache(heads=0), INV), (cache(page=0), INV), (cache(d=0), INV),
    (cache(page=48), UNS), (cache(page=8), UNS), (cache(page=512), UNS), (cache(d=96), UNS), (cache(d=32), UNS), (cache(heads=129), UNS),
    (cache(pages=1 << 28), UNS), (cache(pages=1 << 33), INV), (cache(s_page=1088), 0), (cache(s_page=1072), INV), (cache(s_page=2184), INV),
    (cache(s_head=0), INV), (cache(s_head=1096), INV), (cache(s_head=1 << 40), 0), (cache(pages=1, s_page=0), 0), (cache(heads=1, s_head=0), None),
]


def attn(lib, **over):
    a = dict(ctx=CTX, q=view((1, 4, 5, 64)), c=cache(), table=ADDR, max_pages=4, lens=ADDR, start=ADDR, n=3, bits=None, words=0, out=view((1, 4, 5, 64), data=ADDR + 256), lse=None,
             stream=None)
    a.update(over)
    return lib.sp_tree_attn_q4(*a.values())


def rope(lib, **over):
    freq = (ctypes.c_double * 32)(*[10000.0 ** (-i / 32) for i in range(32)])
    a = dict(ctx=CTX, q=view((1, 4, 5, 64)), k=view((1, 2, 5, 64)), v=view((1, 2, 5, 64)), qw=None, kw=None, eps=1e-6, freq=ctypes.addressof(freq), n=32,
             inter=0, pos=ADDR, qo=view((1, 4, 5, 64)), ko=None, vo=None, c=cache(), slots=ADDR, stream=None)
    a.update(over)
    return lib.sp_qk_norm_rope_q4(*a.values())


def keep(lib, **over):
    a = dict(ctx=CTX, c=cache(), table=ADDR, max_pages=4, past=ADDR + 1024, n=3, kept=ADDR + 2048, n_kept=ADDR + 1280, max_kept=4, lens=ADDR + 4096, stream=None)
    a.update(over)
    return lib.sp_cache_keep_q4(*a.values())


def read(lib, **over):
    a = dict(ctx=CTX, c=cache(), table=ADDR, max_pages=4, lens=ADDR, start=ADDR, n=3, k=view((1, 2, 5, 64)), v=view((1, 2, 5, 64), data=ADDR + 256), stream=None)
    a.update(over)
    return lib.sp_cache_read_q4(*a.values())


@pytest.mark.parametrize("call", [attn, rope, keep, read], ids=["attn", "rope", "keep", "read"])
@pytest.mark.parametrize("i", range(len(BAD_CACHES)))
def test_cache_refusals(lib, call, i):
    c, code = BAD_CACHES[i]
    if code is None or code == 0:                            # valid: without requests nothing is launched
        if call is not rope and code == 0:
            assert call(lib, c=c, n=0) == 0
        return
    assert call(lib, c=c) == code


@pytest.mark.parametrize("over,code", [
    *[(dict(**{k: None}), INV) for k in ("ctx", "q", "table", "lens", "start", "out")],
    (dict(n=-1), INV), (dict(max_pages=0), INV), (dict(n=4097), UNS), (dict(max_pages=1 << 28), UNS), (dict(q=view((1, 4, 5, 64), data=ADDR + 8)), INV),
    (dict(q=view((1, 4, 0, 64))), INV), (dict(q=view((1, 4, 5, 128)), out=view((1, 4, 5, 128), data=ADDR + 256)), INV), (dict(q=view((1, 4, 6, 64))), INV),
    (dict(q=view((1, 4, 5, 64), (0, 320, 64, 2))), INV), (dict(q=view((1, 4, 5, 64), (0, 0, 64, 1))), INV), (dict(q=view((1, 4, 5, 64), (0, 320, 68, 1))), INV),
    (dict(q=view((2, 4, 5, 64)), out=view((2, 4, 5, 64), data=ADDR + 256)), UNS), (dict(q=view((1, 3, 5, 64)), out=view((1, 3, 5, 64), data=ADDR + 256)), UNS),
    (dict(q=view((1, 130, 5, 64)), out=view((1, 130, 5, 64), data=ADDR + 256)), UNS), (dict(bits=ADDR, words=0), UNS), (dict(bits=ADDR, words=9), UNS),
    (dict(out=view((1, 4, 5, 64))), INV),                    # in place
])
def test_attention_refusals(lib, over, code):
    assert attn(lib, **over) == code


_BAD_FREQ = [(ctypes.c_double * 32)(*([x] * 32)) for x in (float("nan"), float("inf"), -1.0, 1e9)]


@pytest.mark.parametrize("over,code", [
    *[(dict(**{k: None}), INV) for k in ("ctx", "q", "k", "v", "pos", "qo", "freq", "slots")], (dict(n=-8), INV), (dict(n=40), UNS), (dict(n=12), UNS),
    *[(dict(freq=ctypes.addressof(f)), INV) for f in _BAD_FREQ], (dict(qw=ADDR), INV), (dict(kw=ADDR), INV), (dict(qw=ADDR + 2, kw=ADDR), INV),
    (dict(qw=ADDR, kw=ADDR, eps=-1.0), INV), (dict(qw=ADDR, kw=ADDR, eps=float("nan")), INV), (dict(ko=view((1, 2, 5, 64))), INV), (dict(vo=view((1, 2, 5, 64))), INV),
    (dict(c=cache(heads=3)), INV), (dict(c=cache(d=128)), INV), (dict(k=view((1, 2, 6, 64)), v=view((1, 2, 6, 64))), INV), (dict(qo=view((1, 4, 6, 64))), INV),
    (dict(v=view((1, 3, 5, 64))), INV), (dict(ko=view((1, 3, 5, 64)), vo=view((1, 3, 5, 64))), INV), (dict(q=view((2, 4, 5, 64)), qo=view((2, 4, 5, 64))), UNS),
])
def test_norm_rope_refusals(lib, over, code):
    assert rope(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    *[(dict(**{k: None}), INV) for k in ("ctx", "table", "past", "kept", "n_kept", "lens")], (dict(n=-1), INV), (dict(max_pages=0), INV), (dict(max_kept=0), INV),
    (dict(n=4097), UNS), (dict(max_pages=1 << 28), UNS), (dict(kept=None, max_kept=-1), INV), (dict(lens=ADDR + 1024), INV), (dict(lens=ADDR + 2048), INV),
    (dict(lens=ADDR + 1280), INV), (dict(lens=ADDR + 16), INV),
])
def test_keep_refusals(lib, over, code):
    assert keep(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    *[(dict(**{k: None}), INV) for k in ("ctx", "table", "lens", "start", "k", "v")], (dict(n=-1), INV), (dict(max_pages=0), INV), (dict(n=4097), UNS),
    (dict(max_pages=1 << 28), UNS), (dict(v=view((1, 2, 5, 64))), INV), (dict(k=view((1, 2, 6, 64))), INV), (dict(c=cache(heads=3)), INV), (dict(c=cache(d=128)), INV),
    (dict(k=view((2, 2, 5, 64)), v=view((2, 2, 5, 64), data=ADDR + 256)), UNS), (dict(k=view((1, 2, 5, 64), (0, 320, 68, 1))), INV), (dict(k=view((1, 2, 0, 64))), INV),
])
def test_read_refusals(lib, over, code):
    assert read(lib, **over) == code


def test_no_requests_is_no_work(lib):
    none = view((1, 4, 0, 64), data=0)
    kv = view((1, 2, 0, 64), data=0)
    assert attn(lib, n=0) == keep(lib, n=0) == read(lib, n=0) == 0
    assert attn(lib, n=0, q=none, out=none, table=None, lens=None, start=None) == read(lib, n=0, k=kv, v=kv, table=None, lens=None, start=None) == 0
    assert keep(lib, n=0, table=None, past=None, kept=None, n_kept=None, lens=None) == 0
    assert attn(lib, n=0, ctx=None) == keep(lib, n=0, ctx=None) == read(lib, n=0, ctx=None) == INV


@pytest.mark.skipif(torch.cuda.is_available(), reason="a valid call would be launched")
def test_valid_calls_without_a_device_are_errors_not_crashes(lib):
    assert attn(lib) == rope(lib) == keep(lib) == read(lib) == -4


def test_page_bytes(lib):
    from paper_2505_19578_b200 import binding
    for d in (64, 128):
        for page in (16, 32, 64, 128, 256):
            assert binding.page_bytes(page, d) == q4.page_bytes(page, d) == page * q4.token_bytes(d)
    for page, d in ((0, 128), (24, 128), (512, 64), (16, 96), (-16, 64)):
        with pytest.raises(binding.SpError, match="-2"):
            binding.page_bytes(page, d)
    assert lib.sp_q4_page_bytes(16, 128, None) == INV


def test_binding_names_what_is_wrong(lib):
    from paper_2505_19578_b200 import binding
    native = binding._decode_calls()
    i = torch.zeros(3, dtype=torch.int32)
    x = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    c = torch.zeros(2, 2, 1088, dtype=torch.uint8)
    for wrong in (c, c.float(), None, 7):
        with pytest.raises(ValueError, match="cache: expected a uint8 tensor on cuda:0"):
            native.cache_keep_q4(0, 0, wrong, i, i, i, i, i, 64, None)
    for name in ("tree_attn_q4", "qk_norm_rope_q4", "cache_read_q4"):
        with pytest.raises(TypeError, match="arguments, got 1"):
            getattr(native, name)(0)
    with pytest.raises(ValueError, match="q: expected a bf16 tensor on cuda:0"):
        native.tree_attn_q4(0, 0, x, c, i, i, i, x, None, None, None)
    with pytest.raises(ValueError, match="q: expected a bf16 tensor on cuda:0"):
        native.qk_norm_rope_q4(0, 0, x, x, x, i, x, x, None, None, c, i, None, None, 1e-6, False, None)
    with pytest.raises(ValueError, match="k_out: expected a bf16 tensor on cuda:0"):
        native.cache_read_q4(0, 0, c, i, i, i, x, x, None)


# ---------------------------------------------------------------- the plain statements

def test_plain_scales_are_the_nearest():
    """Against all 256 scales, for values over the range and beyond, and at exact ties."""
    every = q4.byte_scale(np.arange(256))
    assert np.all(np.diff(every) > 0) and every[0] == q4.LEAST and every[-1] == q4.MOST and np.array_equal(q4.scale_byte(every), np.arange(256))
    rng = np.random.default_rng(0)
    a = np.concatenate([7 * 2.0 ** rng.uniform(-25, 14, 5000), [0.0, 7 * q4.MOST * 2]])
    s, _ = q4.scale_of(a)
    far = np.abs(every[None] - a[:, None] / 7)
    assert np.array_equal(s, every[far.argmin(1)])
    mid = (every[:-1] + every[1:]) / 2 * 7
    assert np.array_equal(q4.scale_of(mid)[0], every[np.arange(1, 256) // 2 * 2])     # ties to the even one


def test_plain_codes_are_the_nearest():
    rng = np.random.default_rng(1)
    x = ref_values(rng, 200, 64)
    codes, s, _ = q4.quantise(x)
    y = q4.values(codes, s)
    step = np.repeat(s, 32, -1)
    assert np.all(np.abs(x - y) <= step / 2) and codes.min() >= 1 and codes.max() <= 15
    codes, s, _ = q4.quantise(np.array([[np.nan, np.inf, -np.inf, 1e30] + [1.0] * 28, [0.0] * 32]))
    assert codes[0, :5].tolist() == [8, 15, 1, 15, 8] and s.tolist() == [[q4.MOST], [q4.LEAST]] and set(codes[1]) == {8}


def ref_values(rng, *shape):
    from tests import _decode_ref as ref
    return ref.bf16_values(rng, *shape)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_plain_layout_is_a_bijection_and_round_trips(d, page):
    """Every half byte of a block belongs to one element of one token, and every byte to one token."""
    owner = np.full(17 * d, -1)
    halves = np.zeros((17 * d, 2), dtype=int)
    for i in range(16):
        k, v, ks, vs, shift = q4.places(i, d)
        for at in (k, v):
            np.add.at(halves, (at, shift // 4), 1)
        for at in (ks, vs):
            halves[at] += 1
        for at in np.unique(np.concatenate([k, v, ks, vs])):
            assert owner[at] == -1
            owner[at] = i
    assert np.all(halves == 1) and np.all(owner >= 0)
    rng = np.random.default_rng(2)
    cache = q4.random_cache(rng, 3, 2, page, d)
    x = [q4.quantise(ref_values(rng, d)) for _ in range(2)]
    q4.put(cache, 1, 0, page - 3, d, *[y[:2] for y in x])
    got = q4.get(cache, 1, 0, page - 3, d)
    whole = q4.unpack(cache, page, d)
    for y, z, w in zip(x, got, whole):
        assert np.array_equal(q4.values(*y[:2]), z) and np.array_equal(w[1, 0, page - 3], z)
