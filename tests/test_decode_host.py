"""The decode-side calls refuse what they do not support, before anything is launched, and the plain statements that the
GPU tests compare with say what they should.  No GPU."""
import ctypes
import struct

import numpy as np
import pytest
import torch

from tests import _decode_ref as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2505_19578_b200 import binding, build
    build.build()
    return binding.load()


INV, UNS = -1, -2
HOST = ctypes.create_string_buffer(1 << 16)                       # stands in for device memory: refused calls touch none
ADDR = (ctypes.addressof(HOST) + 255) & ~255
CTX = ADDR + 4096                                                 # likewise the context, which is read after the checks


def view(shape, stride=None, data=ADDR):
    """An sp_tensor as bytes."""
    if stride is None:
        stride = [shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3], 1]
    return struct.pack("P8q", data, *shape, *stride)


CACHE = (10, 2, 16, 64)


def attn(lib, **over):
    a = dict(ctx=CTX, q=view((1, 4, 5, 64)), kc=view(CACHE), vc=view(CACHE), table=ADDR, max_pages=4, lens=ADDR, start=ADDR, n=3, bits=None, words=0,
             out=view((1, 4, 5, 64)), lse=None, stream=None)
    a.update(over)
    return lib.sp_tree_attn(*a.values())


@pytest.mark.parametrize("over,code", [
    (dict(ctx=None), INV), (dict(q=None), INV), (dict(table=None), INV), (dict(lens=None), INV), (dict(start=None), INV), (dict(out=None), INV),
    (dict(n=-1), INV), (dict(max_pages=0), INV), (dict(n=4097), UNS), (dict(max_pages=1 << 28), UNS),
    (dict(q=view((1, 4, 5, 64), data=ADDR + 8)), INV),                       # alignment
    (dict(q=view((1, 4, 0, 64))), INV), (dict(q=view((1, 4, 5, 128))), INV), (dict(q=view((1, 4, 6, 64))), INV),
    (dict(q=view((1, 4, 5, 64), (0, 320, 64, 2))), INV),                     # inner stride
    (dict(q=view((1, 4, 5, 64), (0, 0, 64, 1))), INV),                       # a broadcast head
    (dict(q=view((1, 4, 5, 64), (0, 320, 68, 1))), INV),                     # rows off the 16-byte grid
    (dict(q=view((2, 4, 5, 64)), out=view((2, 4, 5, 64))), UNS), (dict(q=view((1, 3, 5, 64)), out=view((1, 3, 5, 64))), UNS),
    (dict(q=view((1, 130, 5, 64)), out=view((1, 130, 5, 64))), UNS),
    (dict(kc=view((10, 2, 48, 64)), vc=view((10, 2, 48, 64))), UNS), (dict(kc=view((10, 2, 8, 64)), vc=view((10, 2, 8, 64))), UNS),
    (dict(kc=view((10, 2, 512, 64)), vc=view((10, 2, 512, 64))), UNS), (dict(kc=view((10, 2, 16, 96)), vc=view((10, 2, 16, 96))), UNS),
    (dict(vc=view((9, 2, 16, 64))), INV), (dict(kc=view((1 << 28, 2, 16, 64)), vc=view((1 << 28, 2, 16, 64))), UNS),
    (dict(bits=ADDR, words=0), UNS), (dict(bits=ADDR, words=9), UNS),
])
def test_tree_attn_refusals(lib, over, code):
    assert attn(lib, **over) == code


@pytest.mark.parametrize("pages,s_page,s_head,code", [
    (1 << 26, 2 * 1024 + 8, 1024, UNS),                  # strides with no common divisor but 8: 2^26 x 257 steps
    (1 << 22, 8 * ((1 << 27) + 1), 1024, UNS), (2, 8 * ((1 << 33) + 1), 8 * (1 << 33), UNS),
    (1 << 22, 2 * 1024 + 64, 1024, 0), (1 << 26, 2 * 1024, 1024, 0), (1, 8, 1 << 45, 0), (1 << 26, 64, 1 << 32, 0),
])
def test_tree_attn_cache_strides(lib, pages, s_page, s_head, code):
    """Heads and pages have to fit 31 bits in steps of their strides' greatest common divisor (no request: nothing launched)."""
    c = view((pages, 2, 16, 64), (s_page, s_head, 64, 1))
    assert attn(lib, kc=c, vc=c, n=0 if code == 0 else 3) == code


def rope(lib, **over):
    freq = (ctypes.c_double * 32)(*[10000.0 ** (-i / 32) for i in range(32)])
    a = dict(ctx=CTX, q=view((1, 4, 5, 64)), k=view((1, 2, 5, 64)), v=view((1, 2, 5, 64)), qw=None, kw=None, eps=1e-6, freq=ctypes.addressof(freq), n=32,
             inter=0, pos=ADDR, qo=view((1, 4, 5, 64)), ko=view((1, 2, 5, 64)), vo=view((1, 2, 5, 64)), kc=None, vc=None, slots=None, stream=None)
    a.update(over)
    return lib.sp_qk_norm_rope(*a.values())


_BAD_FREQ = [(ctypes.c_double * 32)(*([x] * 32)) for x in (float("nan"), float("inf"), -1.0, 1e9)]


@pytest.mark.parametrize("over,code", [
    (dict(ctx=None), INV), (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(pos=None), INV), (dict(qo=None), INV),
    (dict(freq=None), INV), (dict(n=-8), INV), (dict(n=40), UNS), (dict(n=12), UNS),
    *[(dict(freq=ctypes.addressof(f)), INV) for f in _BAD_FREQ],
    (dict(qw=ADDR), INV), (dict(kw=ADDR), INV), (dict(qw=ADDR + 2, kw=ADDR), INV), (dict(qw=ADDR, kw=ADDR, eps=-1.0), INV),
    (dict(qw=ADDR, kw=ADDR, eps=float("nan")), INV), (dict(qw=ADDR, kw=ADDR, eps=float("inf")), INV),
    (dict(ko=None), INV), (dict(vo=None), INV), (dict(ko=None, vo=None), INV), (dict(kc=view(CACHE)), INV),
    (dict(kc=view(CACHE), vc=view(CACHE)), INV),                             # no slots
    (dict(kc=view((10, 3, 16, 64)), vc=view((10, 3, 16, 64)), slots=ADDR), INV), (dict(kc=view((10, 2, 16, 128)), vc=view((10, 2, 16, 128)), slots=ADDR), INV),
    (dict(kc=view((10, 2, 24, 64)), vc=view((10, 2, 24, 64)), slots=ADDR), UNS),
    (dict(k=view((1, 2, 6, 64)), v=view((1, 2, 6, 64)), ko=view((1, 2, 6, 64)), vo=view((1, 2, 6, 64))), INV), (dict(qo=view((1, 4, 6, 64))), INV),
    (dict(v=view((1, 3, 5, 64))), INV), (dict(ko=view((1, 3, 5, 64))), INV),
    (dict(q=view((2, 4, 5, 64)), qo=view((2, 4, 5, 64))), UNS),
    (dict(q=view((1, 4, 5, 32)), qo=view((1, 4, 5, 32)), k=view((1, 2, 5, 32)), v=view((1, 2, 5, 32)), ko=view((1, 2, 5, 32)), vo=view((1, 2, 5, 32)), n=16), UNS),
])
def test_norm_rope_refusals(lib, over, code):
    assert rope(lib, **over) == code


def tables(lib, **over):
    a = dict(ctx=CTX, past=ADDR, new=ADDR, n=3, page=16, free=ADDR, n_free=5, table=ADDR, max_pages=4, parents=None, lens=ADDR, start=ADDR, pos=ADDR, slots=ADDR,
             bits=None, words=0, rows=7, info=ADDR, stream=None)
    a.update(over)
    return lib.sp_page_tables(*a.values())


@pytest.mark.parametrize("over,code", [
    *[(dict(**{k: None}), INV) for k in ("ctx", "past", "new", "free", "table", "lens", "start", "pos", "slots", "info")],
    (dict(n=-1), INV), (dict(n_free=-1), INV), (dict(max_pages=0), INV), (dict(rows=-1), INV), (dict(n=4097), UNS), (dict(page=0), UNS), (dict(page=24), UNS),
    (dict(page=8), UNS), (dict(page=512), UNS), (dict(max_pages=1 << 27), UNS), (dict(parents=ADDR), INV), (dict(bits=ADDR), INV),
    (dict(parents=ADDR, bits=ADDR, words=0), UNS), (dict(parents=ADDR, bits=ADDR, words=9), UNS),
])
def test_page_tables_refusals(lib, over, code):
    assert tables(lib, **over) == code


def keep(lib, **over):
    a = dict(ctx=CTX, kc=view(CACHE), vc=view(CACHE), table=ADDR, max_pages=4, past=ADDR, n=3, kept=ADDR, n_kept=ADDR, max_kept=4, lens=ADDR, stream=None)
    a.update(over)
    return lib.sp_cache_keep(*a.values())


@pytest.mark.parametrize("over,code", [
    *[(dict(**{k: None}), INV) for k in ("ctx", "kc", "vc", "table", "past", "kept", "n_kept", "lens")],
    (dict(n=-1), INV), (dict(max_pages=0), INV), (dict(max_kept=0), INV), (dict(n=4097), UNS), (dict(vc=view((10, 1, 16, 64))), INV),
    (dict(kc=view((10, 2, 20, 64)), vc=view((10, 2, 20, 64))), UNS),
])
def test_cache_keep_refusals(lib, over, code):
    assert keep(lib, **over) == code


def test_no_requests_is_no_work(lib):
    assert attn(lib, n=0) == 0 and tables(lib, n=0) == 0 and keep(lib, n=0) == 0


def test_no_requests_need_no_arrays(lib):
    """What a framework hands over for tensors without elements."""
    q = view((1, 4, 0, 64), data=0)
    assert attn(lib, n=0, table=None, lens=None, start=None) == 0 and attn(lib, n=0, q=q, out=q, table=None, lens=None, start=None) == 0
    assert tables(lib, n=0, past=None, new=None, free=None, n_free=0, table=None, lens=None, pos=None, slots=None, rows=0) == 0
    assert keep(lib, n=0, table=None, past=None, kept=None, n_kept=None, lens=None) == 0
    assert attn(lib, n=0, ctx=None) == tables(lib, n=0, ctx=None) == keep(lib, n=0, ctx=None) == INV


@pytest.mark.skipif(torch.cuda.is_available(), reason="a valid call would be launched")
def test_keeping_nothing_is_a_valid_call(lib):
    assert keep(lib, kept=None, max_kept=0) == -4 and keep(lib, kept=None, max_kept=-1) == INV        # without a device: it gets to the launch


@pytest.mark.skipif(torch.cuda.is_available(), reason="a valid call would be launched")
def test_valid_calls_without_a_device_are_errors_not_crashes(lib):
    assert attn(lib) == rope(lib) == tables(lib) == keep(lib) == -4


def test_binding_refuses_what_is_not_on_the_device(lib):
    from paper_2505_19578_b200 import binding
    native = binding._decode_calls()
    i = torch.zeros(3, dtype=torch.int32)
    x = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    for wrong in (i, i.long(), None, 7):
        with pytest.raises(ValueError, match="past_lens: expected a contiguous int32 tensor on cuda:0"):
            native.page_tables(0, 0, wrong, i, 16, i, i, i, i, i, i, i, None, None, None)
    for wrong in (x, x.float(), "q"):
        with pytest.raises(ValueError, match="q: expected a bf16 tensor on cuda:0"):
            native.tree_attn(0, 0, wrong, x, x, i, i, i, x, None, None, None)
        with pytest.raises(ValueError, match="q: expected a bf16 tensor on cuda:0"):
            native.qk_norm_rope(0, 0, wrong, x, x, i, x, x, None, None, None, None, None, None, None, 1e-6, False, None)
    with pytest.raises(ValueError, match="k_cache: expected a bf16 tensor"):
        native.cache_keep(0, 0, x, x, i, i, i, i, i, None)
    with pytest.raises(TypeError, match="expected 10 arguments, got 1"):
        native.cache_keep(0)
    with pytest.raises(OverflowError):
        native.cache_keep(0, 1 << 40, x, x, i, i, i, i, i, None)


# ---------------------------------------------------------------- the plain statements

def test_plain_tables_by_hand():
    table = [[7, -1, -1], [3, 4, -1], [-1, -1, -1]]
    t, lens, start, pos, slots, bits, info = ref.page_tables([3, 32, 0], [2, 1, 3], 16, [9, 5, 6], table, 8, [-1, 0, -1, -1, -1, 0, 0, 0], 1)
    assert t.tolist() == [[7, -1, -1], [3, 4, 9], [5, -1, -1]] and lens == [5, 33, 3] and start == [0, 2, 3, 6]
    assert slots == [7 * 16 + 3, 7 * 16 + 4, 9 * 16, 80, 81, 82, None, None]
    assert pos == [3, 4, 32, 0, 0, 1, None, None]            # request 2: two roots, then a child of the first
    assert [b and b[0] for b in bits] == [1, 3, 1, 1, 2, 5, None, None] and info == [6, 2, 0, 33]


def test_plain_rotation_keeps_length_and_composes():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 3, 16))
    f = [1.0, 0.3, 0.01, 0.0, 2.0, 0.5, 0.25, 0.125]
    for inter in (False, True):
        y, _ = ref.norm_rope(x, None, 0.0, f, inter, [5, 0, 131071])
        np.testing.assert_allclose((y * y).sum(-1), (x * x).sum(-1))
        np.testing.assert_allclose(y[:, 1], x[:, 1])
        z, _ = ref.norm_rope(y, None, 0.0, f, inter, [-5, 0, -131071])
        np.testing.assert_allclose(z, x, atol=1e-9)


def test_plain_attention_of_everything_is_softmax():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 8)), rng.standard_normal((5, 8)), rng.standard_normal((5, 8))
    seen = ref.visible(3, 2)
    out, lse, _ = ref.attention(q, k, v, seen)
    z = q @ k.T / np.sqrt(8)
    z[~seen] = -np.inf
    np.testing.assert_allclose(out, np.exp(z) @ v / np.exp(z).sum(-1, keepdims=True))
    np.testing.assert_allclose(lse, np.log(np.exp(z).sum(-1)))
    assert seen.tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 1, 1]]
