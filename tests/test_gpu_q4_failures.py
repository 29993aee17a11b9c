"""The calls on a 4-bit cache around a wait that has run out: they do nothing until the status has been read, and are right again
afterwards, whatever an unfinished call has left in the counters of shared units.  No GPU fault: the wait is the context's own
self-test, and what an unfinished call leaves is written from the host."""
import ctypes

import numpy as np
import pytest
import torch

from tests import _q4_ref as q4
from tests.test_gpu_decode import binding, clean, i32  # noqa: F401 (binding is a fixture)
from tests.test_gpu_q4 import Step

pytestmark = pytest.mark.gpu

# rows per request of each form: 4 and 16 (units that many CTAs share), 36 and 160 (tiles)
FORMS = pytest.mark.parametrize("n", [1, 4, 9, 40])


def long_step(n, seed=100):
    """Two key heads over 9000 keys: each unit is cut over dozens of CTAs."""
    return Step(seed + n, 8, 2, 128, 32, [(9000, n), (70, 1)], "tree")


def counters(binding, ctx, write=None):  # noqa: F811
    buf, n = (ctypes.c_int32 * 1024)(*(write or [])), ctypes.c_int(1024 if write is None else len(write))
    code = binding.load().sp_internal_split_counters(ctx._h, buf, ctypes.byref(n), int(write is not None))
    assert code == 0
    return list(buf[:n.value])


def time_out(ctx):
    torch.cuda.synchronize()
    ctx.selftest_wait_timeout(200_000)
    torch.cuda.synchronize()


@FORMS
@pytest.mark.parametrize("kernel", ["tc", "simt"])
def test_attention_does_nothing_after_a_timeout_and_is_right_once_it_was_read(binding, kernel, n):  # noqa: F811
    ctx = binding.Context(kernel=kernel)
    s = long_step(n)
    s.call(ctx)
    clean(ctx)
    s.check()
    first = s.out.clone(), s.lse.clone()
    s.blank()
    time_out(ctx)
    for _ in range(2):
        s.call(ctx)
    torch.cuda.synchronize()
    assert bool((s.out == 9).all()) and bool((s.lse == 9).all())
    assert ctx.status() == (binding.SP_ERR_TIMEOUT, 99) and ctx.status() == (0, 0)
    s.call(ctx)
    clean(ctx)
    assert torch.equal(first[0].view(torch.int16), s.out.view(torch.int16)) and torch.equal(first[1], s.lse)


def test_the_other_calls_do_nothing_after_a_timeout(binding):  # noqa: F811
    hkv, d, page = 2, 64, 16
    g = torch.Generator().manual_seed(3)
    ctx = binding.Context()
    before = torch.randint(0, 256, (300, hkv, q4.page_bytes(page, d)), dtype=torch.uint8, generator=g).cuda()
    cache = before.clone()
    table, freq = i32([list(range(300))]), torch.tensor(1e4 ** (-np.arange(32) / 32.0))

    def calls():
        outs = []
        for rows in (3, 4000):                                                # both forms of the append
            x = torch.randn(rows, 4 + 2 * hkv, d, generator=g).to(torch.bfloat16).cuda()
            q, k, v = (y.transpose(0, 1) for y in x.split([4, hkv, hkv], 1))
            outs += [torch.full((h, rows, d), 9.0, dtype=torch.bfloat16, device="cuda") for h in (4, hkv, hkv)]
            ctx.sp_qk_norm_rope_q4(q, k, v, i32(range(rows)), freq, outs[-3], cache, i32(range(rows)), outs[-2], outs[-1])
        lens = i32([-7])
        ctx.sp_cache_keep_q4(cache, table, i32([100]), i32([[3, 8, 70]]), i32([3]), lens, d)
        outs += [torch.full((hkv, 500, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        ctx.sp_cache_read_q4(cache, table, i32([500]), i32([0, 500]), outs[-2], outs[-1])
        torch.cuda.synchronize()
        return outs, lens

    time_out(ctx)
    outs, lens = calls()
    assert all(bool((o == 9).all()) for o in outs) and lens.tolist() == [-7] and torch.equal(cache, before)
    assert ctx.status() == (binding.SP_ERR_TIMEOUT, 99) and ctx.status() == (0, 0)
    outs, lens = calls()
    clean(ctx)
    assert all(not bool((o == 9).any()) for o in outs) and lens.tolist() == [103] and not torch.equal(cache, before)
    k, _ = q4.unpack(cache.cpu().numpy(), page, d)
    assert np.array_equal(outs[-2].float().cpu().numpy().astype(np.float64), k.transpose(1, 0, 2, 3).reshape(hkv, -1, d)[:, :500])


@FORMS
def test_counters_that_an_unfinished_call_left_are_cleared_with_the_timeout(binding, n):  # noqa: F811
    ctx = binding.Context()
    s = long_step(n)
    ctx.reserve_decode()
    size = len(counters(binding, ctx))
    assert size == torch.cuda.get_device_properties(0).multi_processor_count and not any(counters(binding, ctx))
    s.call(ctx)
    clean(ctx)
    s.check()
    assert not any(counters(binding, ctx))                                     # every call leaves them at zero
    first = s.out.clone(), s.lse.clone()
    counters(binding, ctx, [1 + i % 5 for i in range(size)])
    assert counters(binding, ctx) == [1 + i % 5 for i in range(size)]
    time_out(ctx)
    assert ctx.status() == (binding.SP_ERR_TIMEOUT, 99)
    assert not any(counters(binding, ctx))
    s.blank()
    s.call(ctx)
    clean(ctx)
    assert torch.equal(first[0].view(torch.int16), s.out.view(torch.int16)) and torch.equal(first[1], s.lse)
    assert not any(counters(binding, ctx))


def test_counters_are_zero_after_a_bad_page_in_a_shared_unit(binding):  # noqa: F811
    """A range failure stops nobody: every CTA still arrives."""
    ctx = binding.Context()
    for n in (1, 4):
        s = long_step(n, 300)
        s.table_d[0, 5] = 10 ** 6
        s.call(ctx)
        torch.cuda.synchronize()
        assert ctx.status() == (binding.SP_ERR_RANGE, 71) and not any(counters(binding, ctx))
        s.check(skip=(0,))
        t = long_step(n, 301)
        t.call(ctx)
        clean(ctx)
        t.check()


def test_keep_refuses_a_head_dim_that_is_not_the_caches(binding):  # noqa: F811
    """Pages of 16 tokens of 128 elements and of 32 of 64 have the same bytes: with `page` given, they are told apart."""
    ctx = binding.Context()
    table, past, kept, count = i32([[1, 0]]), i32([3]), i32([[1, 4]]), i32([2])
    for page, d, wrong_page, wrong_d in ((16, 128, 32, 64), (64, 64, 32, 128)):
        before = torch.randint(0, 256, (2, 3, q4.page_bytes(page, d)), dtype=torch.uint8).cuda()
        cache, lens = before.clone(), i32([-7])
        with pytest.raises(ValueError, match=f"pages of {q4.page_bytes(page, d)} bytes are not {page} tokens of {wrong_d} elements"):
            ctx.sp_cache_keep_q4(cache, table, past, kept, count, lens, wrong_d, page=page)
        with pytest.raises(ValueError, match="are not"):
            ctx.sp_cache_keep_q4(cache, table, past, kept, count, lens, d, page=wrong_page)
        with pytest.raises(binding.SpError, match="-2"):
            ctx.sp_cache_keep_q4(cache, table, past, kept, count, lens, d, page=24)
        clean(ctx)
        assert torch.equal(cache, before) and lens.tolist() == [-7]
        ctx.sp_cache_keep_q4(cache, table, past, kept, count, lens, d, page=page)
        clean(ctx)
        whole = cache.clone()
        cache.copy_(before)
        ctx.sp_cache_keep_q4(cache, table, past, kept, count, lens, d)
        clean(ctx)
        assert torch.equal(cache, whole) and not torch.equal(cache, before) and lens.tolist() == [5]
