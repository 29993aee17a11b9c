"""What can be done with a prefix in a 4-bit cache: read back whole, it goes through the prefill calls beside its own queries, which have
to be as many; the queries of a chunk behind it go through sp_tree_attn_q4 as a chain."""
import numpy as np
import pytest
import torch

from tests import _decode_ref as ref
from tests import _q4_ref as q4
from tests.test_gpu_decode import binding, clean, dev, host, i32  # noqa: F401 (binding is a fixture)

pytestmark = pytest.mark.gpu


def test_a_prompt_read_back_through_prefill_and_a_chunk_behind_it_as_a_chain(binding):  # noqa: F811
    hq, hkv, d, page, prompt, chunk = 4, 2, 128, 64, 256, 37
    rng = np.random.default_rng(12)
    ctx = binding.Context()
    total = prompt + chunk
    x = ref.bf16_values(rng, total, hq + 2 * hkv, d)
    t = dev(x)
    pages = rng.permutation(-(-total // page) + 1)[: -(-total // page)]
    slots = pages[np.arange(total) // page] * page + np.arange(total) % page
    cache = torch.zeros(int(pages.max()) + 1, hkv, q4.page_bytes(page, d), dtype=torch.uint8, device="cuda")
    freq = torch.tensor(1e4 ** (-np.arange(64) / 64.0))
    q_out = torch.empty(hq, total, d, dtype=torch.bfloat16, device="cuda")
    for lo, hi in ((0, prompt), (prompt, total)):
        q, k, v = (y.transpose(0, 1) for y in t[lo:hi].split([hq, hkv, hkv], 1))
        ctx.sp_qk_norm_rope_q4(q, k, v, i32(np.arange(lo, hi)), freq, q_out[:, lo:hi], cache, i32(slots[lo:hi]))
    table = i32(pages[None])
    ko, vo = (torch.empty(hkv, prompt, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.sp_cache_read_q4(cache, table, i32([prompt]), i32([0, prompt]), ko, vo)
    out = torch.empty(hq, prompt, d, dtype=torch.bfloat16, device="cuda")
    own_q = q_out[:, :prompt].contiguous()
    ctx.sp_dense_pivot_attn(own_q, ko, vo, range(hq), 128, out)
    rest = torch.empty(hq, chunk, d, dtype=torch.bfloat16, device="cuda")
    ctx.sp_tree_attn_q4(q_out[:, prompt:], cache, table, i32([total]), i32([0, chunk]), rest)
    clean(ctx)
    kc, vc = (y[pages].transpose(1, 0, 2, 3).reshape(hkv, -1, d)[:, :total] for y in q4.unpack(cache.cpu().numpy(), page, d))
    assert np.array_equal(host(ko), kc[:, :prompt]) and np.array_equal(host(vo), vc[:, :prompt])
    seen = np.tril(np.ones((total, total), dtype=bool))
    for h in range(hq):
        g = h * hkv // hq
        want, _, tol = ref.attention(host(q_out)[h], kc[g], vc[g], seen)
        assert np.all(np.abs(host(out)[h] - want[:prompt]) <= tol[:prompt]) and np.all(np.abs(host(rest)[h] - want[prompt:]) <= tol[prompt:])
    # fewer queries than keys, or a history that is not a whole number of blocks: the prefill calls have no place for them
    for bad_q, bad_kv in ((own_q[:, 128:], ko), (own_q[:, :200], ko[:, :200])):
        kv = [bad_kv.contiguous(), vo[:, : bad_kv.shape[1]].contiguous()]
        with pytest.raises(binding.SpError):
            ctx.sp_dense_pivot_attn(bad_q.contiguous(), *kv, range(hq), 128, torch.empty_like(bad_q))
        with pytest.raises(binding.SpError):
            ctx.sp_prefill_attn(bad_q.contiguous(), *kv, [0] * hq, [0], 0.9, 128, torch.empty_like(bad_q))
    clean(ctx)
