"""GPU parity: the CUDA library, called through its C ABI, against the float64
oracle on the same seeded bf16 inputs."""
import numpy as np
import pytest
import torch

from oracle import shareprefill_oracle as orc
from paper_2505_19578_b200 import synth
from tests import _parity as par

pytestmark = pytest.mark.gpu

KERNELS = ["tc", "tc1", "simt"]


@pytest.fixture(scope="module")
def binding():
    from paper_2505_19578_b200 import binding as b, build
    build.build()
    return b


def _rand_layer(seed, Hq, Hkv, N, d, scale=2.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    q = (torch.randn(Hq, N, d, generator=g) * scale / d ** 0.25).to(torch.bfloat16)
    k = (torch.randn(Hkv, N, d, generator=g) * scale / d ** 0.25).to(torch.bfloat16)
    v = torch.randn(Hkv, N, d, generator=g).to(torch.bfloat16)
    return q, k, v


def _sync_ok(ctx):
    torch.cuda.synchronize()
    assert ctx.status() == (0, 0)


# ------------------------------------------------------------------ step 1: dense + importance

@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("Hq,Hkv,N,d,B", [(4, 2, 512, 64, 64), (4, 1, 640, 128, 128), (2, 2, 384, 128, 64),
                                          (3, 1, 512, 64, 128), (2, 1, 128, 128, 128)])
def test_dense_pivot_attn_matches_oracle(binding, kernel, Hq, Hkv, N, d, B):
    q, k, v = _rand_layer(1, Hq, Hkv, N, d)
    Q, K, V = par.f64(q), par.f64(k), par.f64(v)
    ctx = binding.Context(kernel=kernel)
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    heads = list(range(Hq))[::-1]            # any order
    Nb = N // B
    out = torch.full_like(qd, float("nan"))
    imp = torch.full((Hq, Nb, Nb), float("nan"), device="cuda")
    lse = torch.full((Hq, N), float("nan"), device="cuda")
    ctx.sp_dense_pivot_attn(qd, kd, vd, heads, B, out, importance_out=imp, lse_out=lse)
    _sync_ok(ctx)
    for t, h in enumerate(heads):
        I, O = orc.importance_map(Q, K, V, h, B)
        par.assert_out_close(par.f64(out[h]), O, f"head {h}")
        got = imp[t].cpu().numpy().astype(np.float64)
        assert np.all(np.triu(got, 1) == 0)
        np.testing.assert_allclose(got, I, rtol=0, atol=par.IMP_ATOL)
        np.testing.assert_allclose(got.sum(axis=1), 1.0, atol=1e-5)
        # log-sum-exp of the scaled logits, natural log
        g = h // (Hq // Hkv)
        S = (Q[h] @ K[g].T) / np.sqrt(d)
        S = np.where(np.tril(np.ones((N, N), bool)), S, -np.inf)
        ref_lse = np.log(np.exp(S - S.max(1, keepdims=True)).sum(1)) + S.max(1)
        np.testing.assert_allclose(lse[t].cpu().numpy(), ref_lse, atol=2e-3)


@pytest.mark.parametrize("kernel", KERNELS)
def test_dense_without_importance_and_strided_views(binding, kernel):
    Hq, Hkv, N, d, B = 4, 2, 256, 128, 128
    q, k, v = _rand_layer(2, Hq, Hkv, N, d)
    # K and V interleaved in one buffer, like a fused QKV projection output: [N, 2*Hkv, d]
    kv = torch.stack([k, v], dim=0).permute(2, 0, 1, 3).contiguous().cuda()   # [N, 2, Hkv, d]
    kd = kv[:, 0].permute(1, 0, 2)                                             # [Hkv, N, d] strided
    vd = kv[:, 1].permute(1, 0, 2)
    ctx = binding.Context(kernel=kernel)
    out = torch.zeros(Hq, N, d, dtype=torch.bfloat16, device="cuda")
    ctx.sp_dense_pivot_attn(q.cuda(), kd, vd, [1, 3], B, out)
    _sync_ok(ctx)
    ref = orc.dense_causal_attention(par.f64(q), par.f64(k), par.f64(v), B=B, heads=[1, 3])
    par.assert_out_close(par.f64(out[1]), ref[0])
    par.assert_out_close(par.f64(out[3]), ref[1])
    assert torch.all(out[0] == 0) and torch.all(out[2] == 0)                   # unlisted heads untouched


# ------------------------------------------------------------------ step 2: importance -> mask

def _mask_case(binding, imp_np, gamma):
    ctx = binding.Context()
    n_maps, nb, _ = imp_np.shape
    imp = torch.from_numpy(imp_np).cuda()
    mask = torch.full((n_maps, nb, nb), 7, dtype=torch.uint8, device="cuda")
    counts = torch.full((n_maps, nb), -5, dtype=torch.int32, device="cuda")
    idx = torch.full((n_maps, nb, nb), -5, dtype=torch.int32, device="cuda")
    ctx.sp_block_mask_from_importance(imp, gamma, mask, counts, idx)
    _sync_ok(ctx)
    g = par.gamma32(gamma)
    for m in range(n_maps):
        M, cnt, lists, infos = orc.block_mask_from_importance(imp_np[m].astype(np.float64), g)
        # the float64 running sum is associated differently on the GPU: a row whose
        # sum passes within 1e-12 of gamma could differ; none of these inputs has one
        for i in range(nb):
            assert min(abs(infos[i]["cum_at_cut"] - g), abs(infos[i]["cum_before_cut"] - g)) > 1e-12 \
                or infos[i]["cum_at_cut"] == g
        assert np.array_equal(mask[m].cpu().numpy(), M)
        assert np.array_equal(counts[m].cpu().numpy(), cnt)
        got_idx = idx[m].cpu().numpy()
        for i in range(nb):
            assert np.array_equal(got_idx[i, :cnt[i]], lists[i])
            assert np.all(got_idx[i, cnt[i]:] == -1)


@pytest.mark.parametrize("nb", [1, 2, 31, 32, 33, 64, 100, 257, 512, 1024])
def test_block_mask_bit_exact_random(binding, nb):
    rng = np.random.default_rng(nb)
    n_maps = 3 if nb <= 257 else 2
    x = rng.random((n_maps, nb, nb)) ** 6
    x = np.tril(x)
    x /= x.sum(axis=2, keepdims=True)
    x = x.astype(np.float32)
    x += np.triu(np.full((nb, nb), 0.5, np.float32), 1)      # junk above the diagonal must be ignored
    for gamma in (0.9, 0.5, 0.999):
        _mask_case(binding, x, gamma)


def test_block_mask_ties_zeros_and_extremes(binding):
    nb = 40
    x = np.zeros((4, nb, nb), np.float32)
    for i in range(nb):
        x[0, i, :i + 1] = 1.0 / (i + 1)                       # all equal: ties -> lowest indices
        x[1, i, :i + 1] = 0.0                                  # all zero: never reaches gamma -> everything
        x[1, i, i // 2] = 0.25
        x[2, i, :i + 1] = np.float32(2.0) ** -np.arange(1, i + 2)   # exact binary fractions
        x[3, i, i] = 1.0                                       # one-hot on the diagonal
    _mask_case(binding, x, 0.75)                               # map 2: 0.5 + 0.25 == 0.75 exactly ('>=')
    _mask_case(binding, x, 0.9)
    _mask_case(binding, x, 1.5)                                # unreachable -> every causal tile
    _mask_case(binding, x, 1e-6)                               # -> the arg-max tile only


# ------------------------------------------------------------------ step 3: block-sparse attention

@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("Hq,Hkv,N,d,B", [(4, 2, 1024, 64, 64), (4, 1, 1536, 128, 128), (2, 2, 768, 128, 64)])
def test_block_sparse_attn_matches_oracle(binding, kernel, Hq, Hkv, N, d, B):
    q, k, v = _rand_layer(3, Hq, Hkv, N, d)
    Q, K, V = par.f64(q), par.f64(k), par.f64(v)
    Nb = N // B
    rng = np.random.default_rng(5)
    n_lists = 2
    masks = np.zeros((n_lists, Nb, Nb), np.uint8)
    for l in range(n_lists):
        m = np.tril(rng.random((Nb, Nb)) < 0.35).astype(np.uint8)
        for i in range(Nb):
            if m[i].sum() == 0:
                m[i, rng.integers(0, i + 1)] = 1               # never the diagonal by construction
        masks[l] = m
    counts = masks.sum(axis=2).astype(np.int32)
    indices = np.full((n_lists, Nb, Nb), -1, np.int32)
    for l in range(n_lists):
        for i in range(Nb):
            sel = np.nonzero(masks[l, i])[0]
            indices[l, i, :len(sel)] = sel
    ctx = binding.Context(kernel=kernel)
    out = torch.full((Hq, N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    heads = [2, 0, 3, 1] if Hq == 4 else [1, 0]
    lists = [1, 0, -1, 1] if Hq == 4 else [-1, 1]              # one head dense (list -1)
    ctx.sp_block_sparse_attn(q.cuda(), k.cuda(), v.cuda(), heads, lists, torch.from_numpy(counts).cuda(),
                             torch.from_numpy(indices).cuda(), B, out)
    _sync_ok(ctx)
    for h, l in zip(heads, lists):
        M = masks[l] if l >= 0 else np.tril(np.ones((Nb, Nb), np.uint8))
        ref = orc.masked_attention(Q, K, V, h, M, B)
        par.assert_out_close(par.f64(out[h]), ref, f"head {h}")


def test_two_heads_of_one_kv_head_share_work_items(binding):
    """Heads of one KV head that walk the same list are given common work items (tile A = a row-block of one head, tile B
    = the same row-block of the other).  Every tile still walks its own list in the same order, so the result is the same
    bit for bit as with one head per item, and it matches the oracle.  11 row-blocks: the odd tail; five heads of one
    KV head on two lists and dense: two pairs and one head left over."""
    Hq, Hkv, N, d, B = 6, 1, 1408, 128, 128
    q, k, v = _rand_layer(17, Hq, Hkv, N, d)
    Q, K, V = par.f64(q), par.f64(k), par.f64(v)
    Nb = N // B
    rng = np.random.default_rng(9)
    masks = np.zeros((2, Nb, Nb), np.uint8)
    for l in range(2):
        m = np.tril(rng.random((Nb, Nb)) < 0.4).astype(np.uint8)
        for i in range(Nb):
            if m[i].sum() == 0:
                m[i, rng.integers(0, i + 1)] = 1
        masks[l] = m
    counts = torch.from_numpy(masks.sum(axis=2).astype(np.int32)).cuda()
    indices = np.full((2, Nb, Nb), -1, np.int32)
    for l in range(2):
        for i in range(Nb):
            sel = np.nonzero(masks[l, i])[0]
            indices[l, i, :len(sel)] = sel
    indices = torch.from_numpy(indices).cuda()
    heads = [4, 0, 3, 5, 1, 2]
    lists = [1, 0, 1, -1, 1, -1]        # list 1: heads 4 and 3 together, head 1 alone; dense: heads 5 and 2 together
    qc, kc, vc = q.cuda(), k.cuda(), v.cuda()
    outs = {}
    for kern in ("tc", "tc_single_head_items"):
        ctx = binding.Context(kernel=kern)
        out = torch.full((Hq, N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        ctx.sp_block_sparse_attn(qc, kc, vc, heads, lists, counts, indices, B, out)
        _sync_ok(ctx)
        outs[kern] = out
    assert torch.equal(outs["tc"], outs["tc_single_head_items"])
    for h, l in zip(heads, lists):
        M = masks[l] if l >= 0 else np.tril(np.ones((Nb, Nb), np.uint8))
        par.assert_out_close(par.f64(outs["tc"][h]), orc.masked_attention(Q, K, V, h, M, B), f"head {h}")
    # dense with the importance map: the three heads 5, 2, 0 of the KV head -> one pair and one head alone
    imps = {}
    for kern in ("tc", "tc_single_head_items"):
        ctx = binding.Context(kernel=kern)
        out = torch.zeros((Hq, N, d), dtype=torch.bfloat16, device="cuda")
        imp = torch.full((3, Nb, Nb), float("nan"), device="cuda")
        ctx.sp_dense_pivot_attn(qc, kc, vc, [5, 2, 0], B, out, importance_out=imp)
        _sync_ok(ctx)
        imps[kern] = (out, imp)
    assert torch.equal(imps["tc"][0], imps["tc_single_head_items"][0])
    assert torch.equal(imps["tc"][1], imps["tc_single_head_items"][1])
    for t, h in enumerate([5, 2, 0]):
        imp_ref, o_ref = orc.importance_map(Q, K, V, h, B)
        par.assert_out_close(par.f64(imps["tc"][0][h]), o_ref, f"dense head {h}")
        np.testing.assert_allclose(imps["tc"][1][t].cpu().numpy(), imp_ref, rtol=0, atol=par.IMP_ATOL)


# ------------------------------------------------------------------ the whole layer

_run_layer = par.run_layer
_check_layer = par.check_layer


@pytest.mark.parametrize("kernel", KERNELS)
def test_prefill_tiny_config_full(binding, kernel):
    L = synth.make_layer(synth.CONFIGS["tiny"], seed=0)
    out, mask = _run_layer(binding, L, 0.9, kernel)
    _check_layer(L, 0.9, out, mask)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("name,seq,gamma", [("llama8b_32k", 4096, 0.9), ("qwen7b_64k", 2048, 0.95),
                                            ("llama8b_128k", 4096, 0.8)])
def test_prefill_model_shapes_reduced_seq(binding, kernel, name, seq, gamma):
    L = synth.make_layer(synth.scaled(synth.CONFIGS[name], seq), seed=1)
    out, mask = _run_layer(binding, L, gamma, kernel)
    _check_layer(L, gamma, out, mask)


def test_prefill_layer_stack_reduced(binding):
    # the layer-stack workload: every layer its own seeded inputs and 3..6 clusters (one pivot each), layers independent
    import dataclasses
    base = synth.scaled(synth.CONFIGS["llama8b_128k"], 2048)
    for layer, n_clusters in enumerate((3, 6, 5, 4)):
        L = synth.make_layer(dataclasses.replace(base, n_clusters=n_clusters), seed=100 + layer)
        assert len(L["pivot_heads"]) == n_clusters
        out, mask = _run_layer(binding, L, 0.9, "tc")
        _check_layer(L, 0.9, out, mask)


@pytest.mark.parametrize("kernel", KERNELS)
def test_prefill_degenerate_head_sets(binding, kernel):
    cfg = synth.scaled(synth.CONFIGS["tiny"], 512)
    L = synth.make_layer(cfg, seed=2)
    # no pivots at all: every head dense
    L0 = dict(L, pivot_heads=[])
    out, mask = _run_layer(binding, L0, 0.9, kernel)
    _check_layer(L0, 0.9, out, mask)
    # every head a pivot
    L1 = dict(L, pivot_heads=list(range(cfg.n_q_heads)))
    out, mask = _run_layer(binding, L1, 0.9, kernel)
    _check_layer(L1, 0.9, out, mask)
    # unclustered heads (-1), a cluster without pivot, two pivots in one cluster (first listed wins)
    cm = [0, 0, 0, 1, 1, -1, 2, 0]
    L2 = dict(L, cluster_map=cm, pivot_heads=[2, 0, 3])
    out, mask = _run_layer(binding, L2, 0.9, kernel)
    _check_layer(L2, 0.9, out, mask)
    # gamma beyond reach: every head effectively dense
    out, mask = _run_layer(binding, L, 1.5, kernel)
    _check_layer(L, 1.5, out, mask)


@pytest.mark.parametrize("name,seq", [("llama8b_32k", 4096), ("tiny", 1024), ("qwen7b_64k", 2048)])
def test_prefill_host_buffers_equal_device_call(binding, name, seq):
    # same kernels on the same bits, only the transfers are pipelined around them: outputs must be identical
    L = synth.make_layer(synth.scaled(synth.CONFIGS[name], seq), seed=4)
    cfg = L["cfg"]
    Nb = cfg.seq // cfg.block
    out_d, mask_d = _run_layer(binding, L, 0.9, "tc")
    _check_layer(L, 0.9, out_d, mask_d)
    ctx = binding.Context()
    hq, hk, hv = (L[x].contiguous().pin_memory() for x in ("q", "k", "v"))
    for rep in range(2):                                       # second call reuses the device copies
        hout = torch.full(hq.shape, float("nan"), dtype=torch.bfloat16).pin_memory()
        hmask = torch.full((cfg.n_q_heads, Nb, Nb), 9, dtype=torch.uint8).pin_memory()
        ctx.sp_prefill_attn_host(hq, hk, hv, L["cluster_map"], L["pivot_heads"], 0.9, cfg.block, hout,
                                 mask_out=hmask if rep == 0 else None)
        _sync_ok(ctx)
        assert torch.equal(hout.view(torch.int16), out_d.cpu().view(torch.int16))
        if rep == 0:
            assert torch.equal(hmask, mask_d.cpu())
    # pageable host memory is accepted too
    pout = torch.empty(hq.shape, dtype=torch.bfloat16)
    ctx.sp_prefill_attn_host(L["q"].contiguous(), L["k"].contiguous(), L["v"].contiguous(), L["cluster_map"],
                             L["pivot_heads"], 0.9, cfg.block, pout)
    _sync_ok(ctx)
    assert torch.equal(pout.view(torch.int16), out_d.cpu().view(torch.int16))


@pytest.mark.parametrize("cm,pivots", [
    ([0, 0, 0, 1, 1, -1, 2, 0], [2, 0, 3]),      # unclustered head, cluster without pivot, two pivots in one cluster
    ([0, 0, 0, 0, 0, 0, 0, 0], [5]),             # a single pivot: nothing is held back
    ([0, 1, 0, 1, 0, 1, 0, 1], []),              # no pivot at all: every head runs dense
    ([0, 1, 2, 3, 0, 1, 2, 3], [3, 2, 1, 0]),    # the last pivot's cluster goes after the other clusters' members
    (None, None),                                # head_dim 128 (paired kernel): pivots reversed, one cluster left without
])
def test_prefill_host_buffers_irregular_cluster_tables(binding, cm, pivots):
    # the host-buffer call orders pivots, clusters and copies differently from the device call; same bits out
    if cm is None:
        L = synth.make_layer(synth.scaled(synth.CONFIGS["llama8b_32k"], 2048), seed=9)
        cm, pivots = L["cluster_map"], list(reversed(L["pivot_heads"]))[:-1]
    else:
        L = synth.make_layer(synth.scaled(synth.CONFIGS["tiny"], 1024), seed=9)
    cfg = L["cfg"]
    Nb = cfg.seq // cfg.block
    L2 = dict(L, cluster_map=cm, pivot_heads=pivots)
    out_d, mask_d = _run_layer(binding, L2, 0.9, "tc")
    _check_layer(L2, 0.9, out_d, mask_d)
    ctx = binding.Context()
    hq, hk, hv = (L[x].contiguous().pin_memory() for x in ("q", "k", "v"))
    hout = torch.full(hq.shape, float("nan"), dtype=torch.bfloat16).pin_memory()
    hmask = torch.full((cfg.n_q_heads, Nb, Nb), 9, dtype=torch.uint8).pin_memory()
    ctx.sp_prefill_attn_host(hq, hk, hv, cm, pivots, 0.9, cfg.block, hout, mask_out=hmask)
    _sync_ok(ctx)
    assert torch.equal(hout.view(torch.int16), out_d.cpu().view(torch.int16))
    assert torch.equal(hmask, mask_d.cpu())


def test_tc_and_simt_kernels_agree_on_importance(binding):
    # two different algorithms for the tile mass (one pass + spilled statistics vs two passes)
    q, k, v = _rand_layer(7, 2, 1, 1024, 128, scale=3.0)
    res = {}
    for kernel in KERNELS:
        ctx = binding.Context(kernel=kernel)
        out = torch.empty(2, 1024, 128, dtype=torch.bfloat16, device="cuda")
        imp = torch.empty(2, 8, 8, device="cuda")
        ctx.sp_dense_pivot_attn(q.cuda(), k.cuda(), v.cuda(), [0, 1], 128, out, importance_out=imp)
        _sync_ok(ctx)
        res[kernel] = imp.cpu().numpy()
    np.testing.assert_allclose(res["tc"], res["simt"], rtol=0, atol=par.IMP_ATOL)
    np.testing.assert_allclose(res["tc1"], res["simt"], rtol=0, atol=par.IMP_ATOL)


# ------------------------------------------------------------------ argument checking (host side)

def test_invalid_arguments_are_rejected(binding):
    ctx = binding.Context()
    q = torch.zeros(4, 256, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 256, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)

    def code(fn):
        with pytest.raises(binding.SpError) as e:
            fn()
        return e.value.code

    assert code(lambda: ctx.sp_dense_pivot_attn(q, k, k, [0], 32, out)) == binding.SP_ERR_UNSUPPORTED      # block
    assert code(lambda: ctx.sp_dense_pivot_attn(q, k, k, [4], 128, out)) == binding.SP_ERR_INVALID_ARG     # head range
    assert code(lambda: ctx.sp_dense_pivot_attn(q[:, :200], k[:, :200], k[:, :200], [0], 128, out[:, :200])) \
        == binding.SP_ERR_UNSUPPORTED                                                                      # ragged seq
    k3 = torch.zeros(3, 256, 128, dtype=torch.bfloat16, device="cuda")
    assert code(lambda: ctx.sp_dense_pivot_attn(q, k3, k3, [0], 128, out)) == binding.SP_ERR_UNSUPPORTED   # 4 % 3
    q96 = torch.zeros(4, 256, 96, dtype=torch.bfloat16, device="cuda")
    k96 = torch.zeros(2, 256, 96, dtype=torch.bfloat16, device="cuda")
    assert code(lambda: ctx.sp_dense_pivot_attn(q96, k96, k96, [0], 128, torch.zeros_like(q96))) == binding.SP_ERR_UNSUPPORTED
    assert code(lambda: ctx.sp_dense_pivot_attn(q, k, k[:, :128], [0], 128, out)) == binding.SP_ERR_INVALID_ARG
    assert code(lambda: ctx.sp_prefill_attn(q, k, k, [0, 0, 1, 1], [0, 0], 0.9, 128, out)) == binding.SP_ERR_INVALID_ARG  # dup
    k_bcast = k[:1].expand(2, 256, 128)                      # one KV head broadcast over two: head stride 0
    assert code(lambda: ctx.sp_dense_pivot_attn(q, k_bcast, k_bcast, [0], 128, out)) == binding.SP_ERR_INVALID_ARG
    assert code(lambda: ctx.sp_prefill_attn(q, k, k, [0, 0, 1, 1], [0], 0.0, 128, out)) == binding.SP_ERR_INVALID_ARG
    imp = torch.zeros(1, 8, 8, device="cuda")
    cnt = torch.zeros(1, 8, dtype=torch.int32, device="cuda")
    idx = torch.zeros(1, 8, 8, dtype=torch.int32, device="cuda")
    assert code(lambda: ctx.sp_block_mask_from_importance(imp, -1.0, None, cnt, idx)) == binding.SP_ERR_INVALID_ARG
    assert code(lambda: ctx.sp_block_sparse_attn(q, k, k, [0], [3], cnt, idx, 128, out)) == binding.SP_ERR_INVALID_ARG
    # nothing was launched and the context is still fine
    ctx.sp_dense_pivot_attn(q, k, k, [], 128, out)
    torch.cuda.synchronize()
    assert ctx.status() == (0, 0)


def test_random_small_shapes_tensor_core_path_agrees_with_cuda_core_path(binding):
    # Odd numbers of row-blocks (a pair with one tile only), single-block sequences, dropped pivots, unclustered
    # heads, thresholds from loose to unreachable: the paired tensor-core kernel (hand-offs through named barriers)
    # against the plain CUDA-core kernel on the same inputs.  Oracle parity at these sizes is covered above; this
    # one is about never disagreeing, and never stalling, on the shapes a layer can throw at the kernel.
    import dataclasses
    import random
    rnd = random.Random(5)
    ctx = binding.Context()
    base = synth.CONFIGS["llama8b_32k"]
    for case in range(24):
        nb = rnd.choice([1, 2, 3, 5, 8, 9, 17, 33])
        hkv = rnd.choice([1, 2, 4])
        hq = hkv * rnd.choice([1, 2, 4])
        cfg = dataclasses.replace(base, seq=nb * 128, n_q_heads=hq, n_kv_heads=hkv, n_clusters=rnd.randint(1, min(4, hq)),
                                  n_heavy=min(base.n_heavy, nb * 128 - 2), name="random")
        L = synth.make_layer(cfg, seed=100 + case, device="cuda")
        cm, piv = list(L["cluster_map"]), list(L["pivot_heads"])
        if rnd.random() < 0.3 and len(piv) > 1:
            piv = piv[:-1]
        if rnd.random() < 0.3:
            cm[rnd.randrange(hq)] = -1
        gamma = rnd.choice([0.5, 0.8, 0.9, 0.99, 1.5])
        res = {}
        for kern in ("tc", "simt"):
            ctx.set_kernel(kern)
            out = torch.full_like(L["q"], float("nan"))
            mask = torch.zeros(hq, nb, nb, dtype=torch.uint8, device="cuda")
            ctx.sp_prefill_attn(L["q"], L["k"], L["v"], cm, piv, gamma, cfg.block, out, mask_out=mask)
            _sync_ok(ctx)
            res[kern] = (out.float(), mask)
        assert not torch.isnan(res["tc"][0]).any(), (case, nb, hq, piv, gamma)
        assert torch.equal(res["tc"][1], res["simt"][1]), (case, nb, hq, piv, gamma)
        assert (res["tc"][0] - res["simt"][0]).abs().max().item() < 2e-2, (case, nb, hq, piv, gamma)


def test_random_lists_heads_and_host_call(binding):
    """Random head subsets, list assignments (repeated lists on one KV head: shared work items; dense heads; several
    lists), densities and lengths: the block-sparse call with two heads per work item is bit-identical to one head per
    item and agrees with the CUDA-core kernel; the host-buffer call of the whole layer is bit-identical to the
    device-pointer call.  (Oracle parity of the same calls is covered above at fixed shapes.)"""
    import dataclasses
    import random
    rnd = random.Random(23)
    ctxs = {kern: binding.Context(kernel=kern) for kern in ("tc", "tc_single_head_items", "simt")}
    base = synth.CONFIGS["llama8b_32k"]
    for case in range(40):
        nb = rnd.choice([1, 2, 3, 5, 8, 9, 17, 33])
        hkv = rnd.choice([1, 2, 4])
        hq = hkv * rnd.choice([1, 2, 4, 8])
        cfg = dataclasses.replace(base, seq=nb * 128, n_q_heads=hq, n_kv_heads=hkv, n_clusters=rnd.randint(1, min(4, hq)),
                                  n_heavy=min(base.n_heavy, nb * 128 - 2), name="random")
        L = synth.make_layer(cfg, seed=500 + case, device="cuda")
        q, k, v = L["q"], L["k"], L["v"]
        g = np.random.default_rng(case)
        n_lists = rnd.randint(1, 3)
        dens = rnd.choice([0.1, 0.3, 0.6, 1.0])
        masks = np.zeros((n_lists, nb, nb), np.uint8)
        for l in range(n_lists):
            m = np.tril(g.random((nb, nb)) < dens).astype(np.uint8)
            for i in range(nb):
                if m[i].sum() == 0:
                    m[i, g.integers(0, i + 1)] = 1
            masks[l] = m
        counts = torch.from_numpy(masks.sum(axis=2).astype(np.int32)).cuda()
        idx = np.full((n_lists, nb, nb), -1, np.int32)
        for l in range(n_lists):
            for i in range(nb):
                sel = np.nonzero(masks[l, i])[0]
                idx[l, i, :len(sel)] = sel
        idx = torch.from_numpy(idx).cuda()
        heads = rnd.sample(range(hq), rnd.randint(1, hq))
        lists = [rnd.choice([-1] + list(range(n_lists))) for _ in heads]
        outs = {}
        for kern, ctx in ctxs.items():
            out = torch.zeros_like(q)
            ctx.sp_block_sparse_attn(q, k, v, heads, lists, counts, idx, cfg.block, out)
            _sync_ok(ctx)
            outs[kern] = out
        what = (case, nb, hq, hkv, heads, lists)
        assert torch.equal(outs["tc"], outs["tc_single_head_items"]), what
        assert (outs["tc"].float() - outs["simt"].float()).abs().max().item() < 2e-2, what
        cm, piv = list(L["cluster_map"]), list(L["pivot_heads"])
        if rnd.random() < 0.3 and len(piv) > 1:
            piv = piv[:-1]
        if rnd.random() < 0.3:
            cm[rnd.randrange(hq)] = -1
        gamma = rnd.choice([0.5, 0.9, 0.99])
        ctx = ctxs["tc"]
        o_dev = torch.zeros_like(q)
        ctx.sp_prefill_attn(q, k, v, cm, piv, gamma, cfg.block, o_dev)
        _sync_ok(ctx)
        ho = torch.zeros(q.shape, dtype=q.dtype).pin_memory()
        ctx.sp_prefill_attn_host(q.cpu().pin_memory(), k.cpu().pin_memory(), v.cpu().pin_memory(), cm, piv, gamma,
                                 cfg.block, ho)
        _sync_ok(ctx)
        assert torch.equal(ho, o_dev.cpu()), what


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("rise", [9.0, 40.0])
def test_dense_logits_that_climb_within_a_tile(binding, kernel, rise):
    """Every 32 keys the row maximum grows: references move in each chunk of a tile, with sums of earlier tiles and
    weights of the chunk before just written."""
    Hq, Hkv, N, d, B = 4, 2, 640, 128, 128
    q, k, v = _rand_layer(17, Hq, Hkv, N, d)
    q[..., 0] = 8.0
    k[..., 0] = (torch.arange(N) // 32 * (rise * d ** 0.5 / 8)).to(torch.bfloat16)
    ctx = binding.Context(kernel=kernel)
    out = torch.zeros_like(q, device="cuda")
    ctx.sp_dense_pivot_attn(q.cuda(), k.cuda(), v.cuda(), list(range(Hq)), B, out)
    _sync_ok(ctx)
    ref = orc.dense_causal_attention(par.f64(q), par.f64(k), par.f64(v), B=B, heads=list(range(Hq)))
    for h in range(Hq):
        par.assert_out_close(par.f64(out[h]), ref[h], f"head {h}")
