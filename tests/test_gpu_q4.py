"""The operators of the 4-bit cache on the GPU against plain float64 statements: small sizes at which they can go wrong."""
import random

import numpy as np
import pytest
import torch

from tests import _decode_ref as ref
from tests import _q4_ref as q4
from tests.test_gpu_decode import ATTN, binding, clean, dev, host, i32, tree  # noqa: F401 (binding is a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["tc", "simt"])
def attn_ctx(binding, request):  # noqa: F811
    return binding.Context(kernel=request.param)


def u8(x, pad=0):
    """On the device; `pad`: that many bytes between heads and again between pages (multiples of 16)."""
    t = torch.tensor(x)
    if not pad:
        return t.cuda()
    n, h, b = t.shape
    out = torch.full((n, h * (b + pad) + pad), 0xA5, dtype=torch.uint8, device="cuda")
    view = out[:, : h * (b + pad)].unflatten(1, (h, b + pad))[:, :, :b]
    view.copy_(t)
    return view


# ---------------------------------------------------------------- norm, rotation, quantisation

def same_codes(got, x, exact):
    """got: stored values [rows, d]; x: exact ones.  The nearest codes and scales; either neighbour within `exact` steps of a border."""
    codes, s, border = q4.quantise(x)
    want = q4.values(codes, s)
    sure = border > exact
    # a scale next to its border decides all of its group
    sure = (sure.reshape(*sure.shape[:-1], -1, 32) & (q4.scale_of(np.abs(np.nan_to_num(x, nan=0, posinf=1e300, neginf=-1e300)).reshape(*sure.shape[:-1], -1, 32).max(-1))[1]
                                                     > exact)[..., None]).reshape(sure.shape)
    assert np.array_equal(got[sure], want[sure]), (np.argwhere((got != want) & sure)[:5], got[(got != want) & sure][:5], want[(got != want) & sure][:5])
    step = np.repeat(s, 32, -1)
    assert np.all(np.abs(got - want) <= 1.0001 * step)
    return float(np.mean(~sure))


def rope_case(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, pad=0, seed=0, scale=1.0, change=None, eps=1e-6, top=131072):  # noqa: F811
    rng = np.random.default_rng(seed)
    qkv = ref.bf16_values(rng, rows, hq + 2 * hkv, d, scale=scale)
    if change is not None:
        change(qkv, rng)
    weights = [ref.bf16_values(rng, d) if norm else None for _ in range(2)]
    freq = 5e5 ** (-np.arange(n_freq) * 2.0 / max(1, 2 * n_freq))
    pos = rng.integers(0, top, rows)
    pos[: min(rows, 2)] = [0, 1][: min(rows, 2)]
    t = dev(qkv)
    q, k, v = (x.transpose(0, 1) for x in t.split([hq, hkv, hkv], 1))
    make = lambda h: torch.full((h, rows, d), 7.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q_out, k_out, v_out = make(hq), *((make(hkv), make(hkv)) if outs else (None, None))
    pages = -(-rows // page) + 2
    before = rng.integers(0, 256, (pages, hkv, q4.page_bytes(page, d)), dtype=np.uint8)
    cache = u8(before, pad)
    slots = rng.permutation(pages * page)[:rows]
    if rows > 3:
        slots[rng.random(rows) < 0.2] = -1
    ctx = binding.Context()
    ctx.sp_qk_norm_rope_q4(q, k, v, i32(pos), torch.tensor(freq, dtype=torch.float64), q_out, cache, i32(slots), k_out, v_out,
                           None if not norm else dev(weights[0]), None if not norm else dev(weights[1]), eps, interleaved)
    clean(ctx)
    x = qkv.transpose(1, 0, 2)
    with np.errstate(all="ignore"):
        wq, eq = ref.norm_rope(x[:hq], weights[0], eps, freq, interleaved, pos)
        wk, ek = ref.norm_rope(x[hq:hq + hkv], weights[1], eps, freq, interleaved, pos)
        wv = x[hq + hkv:]
        if change is None:
            assert np.all(np.abs(host(q_out) - wq) <= eq + ref.EPS_BF16 * np.abs(wq))
            if outs:
                assert np.all(np.abs(host(k_out) - wk) <= ek + ref.EPS_BF16 * np.abs(wk)) and np.array_equal(host(v_out), wv)
    after = cache.cpu().numpy()
    kc, vc = (c.transpose(0, 2, 1, 3).reshape(-1, hkv, d) for c in q4.unpack(after, page, d))
    used = slots >= 0
    # float64 angles at position 2^17: 2^-36 rad; 16 roundings otherwise: far below 1e-9 of a step of seven to a group
    same_codes(kc[slots[used]], wk.transpose(1, 0, 2)[used], 1e-9)
    same_codes(vc[slots[used]], wv.transpose(1, 0, 2)[used], 0 if change is None else 1e-9)
    for s in slots[used]:                                    # nothing else was written: put the written tokens' bytes back
        k_at, v_at, ks, vs, _ = q4.places(s % page % 16, d)
        for at in (k_at, v_at, ks, vs):
            at = at + s % page // 16 * 17 * d
            after[s // page][:, at] = before[s // page][:, at]
    assert np.array_equal(after, before)
    if pad:
        gaps = cache._base if cache._base is not None else cache
        assert int((gaps == 0xA5).sum()) >= pages * (hkv + 1) * pad


@pytest.mark.parametrize("hq,hkv,d,rows,n_freq,interleaved,norm,outs,page,pad", [
    (32, 8, 128, 1, 64, False, False, False, 64, 0), (32, 8, 128, 1, 64, False, True, True, 16, 0), (28, 4, 128, 37, 64, False, True, True, 16, 16),
    (8, 8, 64, 129, 32, False, True, False, 32, 0), (8, 8, 64, 5, 32, True, True, True, 16, 32), (7, 1, 128, 3, 32, False, False, True, 128, 0),
    (5, 5, 64, 2, 8, True, False, True, 256, 0), (3, 1, 64, 70, 16, False, True, True, 64, 0), (16, 2, 128, 40, 8, False, False, False, 64, 0),
    (16, 3, 128, 40, 24, False, True, False, 64, 0), (4, 2, 128, 33, 56, False, False, False, 16, 0), (6, 6, 64, 20, 24, False, True, True, 16, 0),
    (128, 128, 128, 2, 64, False, True, True, 16, 0), (1, 1, 64, 1, 0, False, True, True, 16, 0), (4, 2, 128, 9, 0, False, False, True, 32, 0),
    # the streaming form
    (16, 2, 128, 1000, 64, True, True, True, 128, 0), (2, 1, 128, 6000, 64, False, True, True, 16, 0), (8, 2, 128, 2369, 64, False, False, False, 64, 48),
    (24, 8, 64, 3001, 16, False, True, True, 32, 0), (8, 4, 128, 3000, 0, False, False, False, 16, 0), (8, 4, 64, 3000, 8, False, False, False, 16, 0)])
def test_norm_rope(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, pad):  # noqa: F811
    rope_case(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, pad)


@pytest.mark.parametrize("rows", [5, 3000])
@pytest.mark.parametrize("scale", [2.0 ** 12, 2.0 ** -18, 2.0 ** -25, 2.0 ** 70], ids=["above the scales", "smallest scales", "below them", "squares past fp32"])
@pytest.mark.parametrize("norm", [False, True])
def test_norm_rope_of_tiny_and_huge_values(binding, scale, norm, rows):  # noqa: F811
    """(bf16 results are checked elsewhere: sums of squares past fp32 are this form's alone.)"""
    rope_case(binding, 4, 2, 128, rows, 64, False, norm, False, 16, seed=3, scale=scale, change=lambda x, r: None)
    if norm:
        rope_case(binding, 2, 2, 64, rows, 32, True, True, False, 16, seed=4, scale=scale, change=lambda x, r: None, eps=0.0)


def test_norm_rope_groups_of_zeros_and_of_one_large_element(binding):  # noqa: F811
    def change(x, rng):
        x[::3] = 0
        x[1::3, :, ::32] *= 64
        x[2::3, :, 5] = 2.0 ** -130
    for norm in (False, True):
        rope_case(binding, 4, 2, 128, 90, 64, False, norm, False, 32, seed=5, change=change)


def test_norm_rope_borders_at_position_zero(binding):  # noqa: F811
    """Nothing turns at position 0: codes and scales lie on borders as often as bf16's few bits make them, and ties are even."""
    def change(x, rng):
        x[:] = np.round(x * 8) / 8
    rope_case(binding, 4, 4, 128, 300, 64, False, False, False, 32, seed=6, change=change, top=1)
    rope_case(binding, 4, 4, 64, 3000, 32, True, False, False, 32, seed=7, change=change, top=1)


@pytest.mark.parametrize("rows", [3, 3000])
def test_norm_rope_of_nan_and_infinity(binding, rows):  # noqa: F811
    """A NaN is stored as 0, an infinity as 7 times its scale; other heads are not touched, and bf16 outputs keep them."""
    hkv, d, page = 3, 128, 16
    rng = np.random.default_rng(8)
    x = ref.bf16_values(rng, rows, 1 + 2 * hkv, d)
    x[0, 2, 7], x[0, 2, 40], x[1, 5, 3], x[1, 5, 90], x[2, 4, :] = np.nan, np.inf, -np.inf, np.nan, np.nan
    t = dev(x)
    q, k, v = (y.transpose(0, 1) for y in t.split([1, hkv, hkv], 1))
    pages = -(-rows // page)
    cache = torch.zeros(pages, hkv, q4.page_bytes(page, d), dtype=torch.uint8, device="cuda")
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    ctx = binding.Context()
    ctx.sp_qk_norm_rope_q4(q, k, v, i32([0] * rows), torch.zeros(0, dtype=torch.float64), torch.empty_like(q), cache, i32(range(rows)), ko, vo)
    clean(ctx)
    kc, vc = (c.transpose(0, 2, 1, 3).reshape(-1, hkv, d) for c in q4.unpack(cache.cpu().numpy(), page, d))
    same_codes(kc[:rows], x[:, 1:1 + hkv], 0)
    same_codes(vc[:rows], x[:, 1 + hkv:], 0)
    assert kc[0, 1, 7] == 0 and kc[0, 1, 40] == 7 * q4.MOST and vc[1, 1, 3] == -7 * q4.MOST and np.all(vc[2, 0] == 0)
    assert torch.equal(torch.isnan(ko), torch.isnan(k)) and torch.equal(torch.isinf(vo), torch.isinf(v))


def test_norm_rope_far_positions(binding):  # noqa: F811
    """Angles at any 32-bit position: within two steps of what float64 gives, which is 2^-21 rad off there itself."""
    hkv, d = 4, 128
    rng = np.random.default_rng(9)
    rows = 200
    x = ref.bf16_values(rng, rows, 1 + 2 * hkv, d)
    freq = 5e5 ** (-np.arange(64) / 64.0)
    pos = rng.integers(2 ** 30, 2 ** 31, rows)
    t = dev(x)
    q, k, v = (y.transpose(0, 1) for y in t.split([1, hkv, hkv], 1))
    cache = torch.zeros(13, hkv, q4.page_bytes(16, d), dtype=torch.uint8, device="cuda")
    ctx = binding.Context()
    ctx.sp_qk_norm_rope_q4(q, k, v, i32(pos), torch.tensor(freq), torch.empty_like(q), cache, i32(range(rows)))
    clean(ctx)
    kc, _ = (c.transpose(0, 2, 1, 3).reshape(-1, hkv, d) for c in q4.unpack(cache.cpu().numpy(), 16, d))
    want, _ = ref.norm_rope(x[:, 1:1 + hkv].transpose(1, 0, 2), None, 0, freq, False, pos)
    same_codes(kc[:rows], want.transpose(1, 0, 2), 1e-4)


def test_norm_rope_is_the_same_in_both_forms_and_in_any_batch(binding):  # noqa: F811
    """A token's codes do not depend on the kernel that stored it."""
    hkv, d, page, rows = 2, 128, 16, 4000
    g = torch.Generator().manual_seed(1)
    x = torch.randn(rows, 4 + 2 * hkv, d, generator=g).to(torch.bfloat16).cuda()
    w = (1 + 0.3 * torch.randn(2, d, generator=g)).to(torch.bfloat16).cuda()
    pos = torch.randint(0, 131072, (rows,), generator=g, dtype=torch.int32).cuda()
    freq = torch.tensor(5e5 ** (-np.arange(64) / 64.0))
    ctx = binding.Context()
    caches = [torch.zeros(rows // page, hkv, q4.page_bytes(page, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    for cache, step in zip(caches, (rows, 13)):
        for lo in range(0, rows, step):
            q, k, v = (y.transpose(0, 1) for y in x[lo:lo + step].split([4, hkv, hkv], 1))
            ctx.sp_qk_norm_rope_q4(q, k, v, pos[lo:lo + step].contiguous(), freq, torch.empty_like(q), cache, i32(range(lo, min(lo + step, rows))), q_weight=w[0], k_weight=w[1])
    clean(ctx)
    assert torch.equal(*caches)


def test_norm_rope_in_place_on_another_stream_and_captured(binding):  # noqa: F811
    hkv, d, page, rows = 2, 128, 32, 50
    rng = np.random.default_rng(5)
    freq = 5e5 ** (-np.arange(64) / 64.0)
    ctx = binding.Context()
    s = torch.cuda.Stream()
    t = torch.empty(rows, 8 + 2 * hkv, d, dtype=torch.bfloat16, device="cuda")
    pos_d, slots = i32([0] * rows), i32(range(rows))
    cache = torch.zeros(2, hkv, q4.page_bytes(page, d), dtype=torch.uint8, device="cuda")
    q, k, v = (y.transpose(0, 1) for y in t.split([8, hkv, hkv], 1))
    call = lambda **kw: ctx.sp_qk_norm_rope_q4(q, k, v, pos_d, torch.tensor(freq), q, cache, slots, k, v, **kw)  # noqa: E731
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for how in ("stream", "graph", "graph"):
        x = ref.bf16_values(rng, rows, 8 + 2 * hkv, d)
        pos = rng.integers(0, 131072, rows)
        t.copy_(dev(x))
        pos_d.copy_(i32(pos))
        cache.zero_()
        torch.cuda.synchronize()
        if how == "stream":
            call(stream=s)
        else:
            graph.replay()
        clean(ctx)
        x = x.transpose(1, 0, 2)
        want, err = ref.norm_rope(x[:10], None, 0, freq, False, pos)
        assert np.all(np.abs(host(t).transpose(1, 0, 2)[:10] - want) <= err + ref.EPS_BF16 * np.abs(want)) and np.array_equal(host(v), x[10:])
        kc, vc = (c.transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:rows] for c in q4.unpack(cache.cpu().numpy(), page, d))
        same_codes(kc, want[8:].transpose(1, 0, 2), 1e-9)
        same_codes(vc, x[10:].transpose(1, 0, 2), 0)


@pytest.mark.parametrize("rows", [3, 4000])
def test_norm_rope_slot_behind_the_cache_is_reported_not_followed(binding, rows):  # noqa: F811
    ctx = binding.Context()
    x = torch.randn(rows, 4, 64, device="cuda").to(torch.bfloat16)
    whole = torch.zeros(4, 1, q4.page_bytes(16, 64), dtype=torch.uint8, device="cuda")
    cache = whole[1:3]
    q, k, v = x[:, :2].transpose(0, 1), x[:, 2:3].transpose(0, 1), x[:, 3:].transpose(0, 1)
    slots = i32([31] + [32, 2 ** 31 - 1] + [-1] * (rows - 3))
    ctx.sp_qk_norm_rope_q4(q, k, v, i32(range(rows)), torch.ones(0, dtype=torch.float64), torch.empty_like(q), cache, slots)
    torch.cuda.synchronize()
    assert ctx.status() == (binding.SP_ERR_RANGE, 76) and ctx.status() == (0, 0)
    _, vc = q4.unpack(cache.cpu().numpy(), 16, 64)
    same_codes(vc[1, 0, 15:], host(x[:1, 3]), 0)
    assert int((whole[0] != 0).sum()) == int((whole[3] != 0).sum()) == 0 and np.all(vc[0] == -8 * q4.LEAST)


# ---------------------------------------------------------------- attention over the cache

class Step:
    """Inputs of one call, host copies beside them."""

    def __init__(self, seed, hq, hkv, d, page, reqs, kind="chain", pad=0, gap=0, scale=1.0):
        r, rng = random.Random(seed), np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.page, self.reqs = hq, hkv, d, page, reqs
        rows = sum(n for _, n in reqs) + pad
        self.rows = rows
        self.q = ref.bf16_values(rng, rows, hq, d, scale=scale)
        need = [-(-(p + n) // page) for p, n in reqs]
        width = max(max(need), 1) + 1
        total = sum(need) + 2
        order = list(range(total))
        r.shuffle(order)
        self.table = np.full((len(reqs), width), 2 ** 31 - 1)              # entries behind the last page are not read
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.cache = q4.random_cache(rng, total, hkv, page, d, 0.25)        # codes are uniform: values of about 1
        used = np.zeros((total, page), dtype=bool)
        for b, (p, n) in enumerate(reqs):
            for x in range(p + n):
                used[self.table[b, x // page], x % page] = True
        blocks = self.cache.reshape(total, hkv, page // 16, 17 * d)
        for i in range(16):                                                # unused places hold the largest numbers there are
            k, v, ks, vs, _ = q4.places(i, d)
            for pg, blk in np.argwhere(~used[:, i::16]):
                for where, what in ((k, 0), (v, 0), (ks, 255), (vs, 255)):
                    blocks[pg, :, blk, where] = what
        self.k, self.v = q4.unpack(self.cache, page, d)
        self.bits = None
        if kind != "chain":
            words = -(-max(n for _, n in reqs) // 32)
            self.bits = np.zeros((rows, words), dtype=np.int64)
            t = 0
            for p, n in reqs:
                parents = tree(r, n)
                seen = []
                for j in range(n):
                    s = (seen[parents[j]] if parents[j] >= 0 else 0) | 1 << j
                    seen.append(s)
                    if kind == "any":                                      # any bits at all, some rows none
                        s = r.getrandbits(n) if j % 3 else 0
                    for w in range(words):
                        self.bits[t + j, w] = (s >> (32 * w)) & 0xFFFFFFFF
                t += n
            self.bits[t:] = 0xFFFFFFFF
        self.cd = u8(self.cache, gap)
        self.upload()
        self.out = torch.full((rows, hq, d), 9.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
        self.lse = torch.full((hq, rows), 9.0, device="cuda")
        self.lens_d, self.start_d = i32([p + n for p, n in reqs]), i32(np.cumsum([0] + [n for _, n in reqs]))
        self.table_d = i32(self.table)
        self.bits_d = None if self.bits is None else torch.tensor(self.bits).to(torch.int32).cuda()

    def upload(self):
        self.qd = dev(self.q).transpose(0, 1)

    def blank(self):
        self.out.fill_(9)
        self.lse.fill_(9)

    def call(self, ctx, **kw):
        ctx.sp_tree_attn_q4(self.qd, self.cd, self.table_d, self.lens_d, self.start_d, self.out, tree_mask=self.bits_d, lse_out=self.lse, **kw)

    def reference(self):
        t = 0
        for b, (p, n) in enumerate(self.reqs):
            if n == 0:
                continue
            ids = self.table[b, :-(-(p + n) // self.page)]
            k, v = (c[ids].transpose(1, 0, 2, 3).reshape(self.hkv, -1, self.d)[:, :p + n] for c in (self.k, self.v))
            seen = ref.visible(n, p, None if self.bits is None else self.bits[t:t + n].tolist())
            for h in range(self.hq):
                g = h * self.hkv // self.hq
                yield (h, slice(t, t + n), *ref.attention(self.q[t:t + n, h], k[g], v[g], seen))
            t += n

    def check(self, skip=()):
        out, lse = host(self.out), self.lse.cpu().numpy().astype(np.float64)
        with np.errstate(all="ignore"):
            for h, rows, want, want_lse, tol in self.reference():
                if rows.start in skip:
                    continue
                got, got_lse = out[h, rows], lse[h, rows]
                fine = np.isfinite(want)
                assert np.array_equal(fine, np.isfinite(got)), (h, rows)
                far = np.abs(got - want)[fine] - tol[fine]
                assert np.all(far <= 0), (h, rows, float(far.max()), float(np.abs(got - want)[fine].max()))
                f = np.isfinite(want_lse)
                assert np.array_equal(f, np.isfinite(got_lse)) and np.array_equal(np.isnan(want_lse), np.isnan(got_lse))
                # logits within 2^-12 (see the oracle), and one fp32 rounding of the result
                assert np.all(np.abs(got_lse - want_lse)[f] <= 2.0 ** -11 + 2.0 ** -20 * np.abs(want_lse[f]))
        end = sum(n for _, n in self.reqs)
        assert np.all(out[:, end:] == 9) and np.all(lse[:, end:] == 9)        # rows behind the last request: as they were


MORE = [
    # lengths around a block, one row a head; three and four tiles of rows; units cut over warps, CTAs and runs
    (4, 2, 128, 16, [(n, 1) for n in (0, 1, 14, 15, 16, 17, 30, 31, 32, 33, 127, 4000)], "chain", 2, 0),
    (8, 1, 64, 64, [(n, 1) for n in (0, 1, 14, 15, 16, 17, 511, 512, 513)], "chain", 0, 16),
    (1, 1, 128, 128, [(40000, 1)], "chain", 0, 0), (2, 2, 64, 16, [(30000, 2)], "chain", 0, 0),
    (4, 1, 128, 64, [(9000, 4)], "tree", 0, 0), (12, 4, 128, 32, [(5000, 7), (20, 3)], "tree", 1, 32), (4, 1, 128, 256, [(7000, 8), (100, 6), (33, 7)], "tree", 0, 0),
    (4, 1, 64, 16, [(6000, 33), (10, 2), (0, 200)], "any", 3, 0), (3, 1, 128, 16, [(2000, 5)] * 9, "tree", 0, 0), (5, 1, 128, 16, [(1000, 1), (70, 3)] * 20, "chain", 0, 0),
]


@pytest.mark.parametrize("case", [c[:7] + (0,) for c in ATTN] + MORE, ids=[str(i) for i in range(len(ATTN) + len(MORE))])
def test_tree_attn(attn_ctx, case):
    hq, hkv, d, page, reqs, kind, pad, gap = case
    s = Step(len(reqs) + hq, hq, hkv, d, page, reqs, kind, pad, gap)
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()
    first = s.out.clone(), s.lse.clone()
    s.call(attn_ctx)                                                          # the same bits again
    clean(attn_ctx)
    assert torch.equal(first[0].view(torch.int16), s.out.view(torch.int16)) and torch.equal(first[1], s.lse)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 8, 9, 17, 33, 64, 256, 257])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_tree_attn_row_counts(attn_ctx, n, d, page):
    """Rows per request around every change of form: full requests beside short and empty ones."""
    s = Step(n, 4, 2, d, page, [(1500, n), (0, min(n, 5)), (0, 0), (129, 1)], "tree" if n <= 256 else "chain", 1)
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()


def climb(s, step):
    """Keys along q, longer from block to block: each block's logits are `step` nats above the last one's."""
    s.q[:] = np.abs(s.q) + 0.5                                                # rows look the same way
    s.upload()
    s.q[:] = host(s.qd).transpose(1, 0, 2)                                    # (what bf16 made of them)
    blocks = s.cache.reshape(len(s.cache), s.hkv, s.page // 16, 17 * s.d)
    for b, (p, n) in enumerate(s.reqs):
        for x in range(p + n):
            i, blk = x % 16, x % s.page // 16
            k, _, ks, _, shift = q4.places(i, s.d)
            want = step * (x // 16) / (1.3 * s.d ** 0.5 * 4)                   # codes of 12: the value is 4 s, q about 1.3
            byte = q4.scale_byte(q4.scale_of(np.array(abs(want) * 7))[0])
            code = 12 if step > 0 else 4
            at = blocks[s.table[b, x // s.page], :, blk]
            at[:, k] = code * 0x11
            at[:, ks] = byte
    s.k, s.v = q4.unpack(s.cache, s.page, s.d)
    s.cd = u8(s.cache)


@pytest.mark.parametrize("step", [1.0, -1.0, 20.0])
@pytest.mark.parametrize("hq,hkv,d,page,reqs", [(4, 2, 128, 16, [(400, 2), (30, 1)]), (4, 1, 64, 64, [(500, 4), (90, 3)]), (8, 2, 128, 32, [(600, 8)]), (4, 1, 64, 16, [(400, 30)])])
def test_tree_attn_logits_that_climb(attn_ctx, hq, hkv, d, page, reqs, step):
    s = Step(17, hq, hkv, d, page, reqs, "chain")
    climb(s, step)
    s.call(attn_ctx)
    clean(attn_ctx)
    out, lse = host(s.out), s.lse.cpu().numpy()
    for h, rows, want, want_lse, tol in s.reference():
        # (no value in use is above 2)  Logits up to L are off by d 2^-24 L from the products' sums and 2 * 2^-24 L from the scaling: that much of every weight
        off = (d + 2) * 2.0 ** -24 * max(1.0, float(np.abs(want_lse).max()))
        assert np.all(np.abs(out[h, rows] - want) <= tol + 2 * off * 2.0) and np.all(np.abs(lse[h, rows] - want_lse) <= 2.0 ** -11 + off)


def test_tree_attn_lengths_shorter_than_the_new_tokens(attn_ctx):
    """seq_lens below the number of rows: the first rows see nothing and come out as zeros."""
    s = Step(5, 4, 2, 64, 16, [(0, 6)], "chain")
    s.lens_d.fill_(4)
    s.call(attn_ctx)
    clean(attn_ctx)
    out, lse = host(s.out), s.lse.cpu().numpy()
    k, v = (c[s.table[0, :1]].transpose(1, 0, 2, 3).reshape(2, -1, 64)[:, :4] for c in (s.k, s.v))
    seen = np.array([[x + 2 <= j for x in range(4)] for j in range(6)])
    for h in range(4):
        want, want_lse, tol = ref.attention(s.q[:, h], k[h // 2], v[h // 2], seen)
        assert np.all(np.abs(out[h] - want) <= tol) and np.all(out[h, :2] == 0) and np.all(np.isneginf(lse[h, :2]))
    s.lens_d.fill_(0)
    s.call(attn_ctx)
    clean(attn_ctx)
    assert np.all(host(s.out) == 0) and bool(torch.isneginf(s.lse).all())


def test_tree_attn_of_queries_that_are_not_finite(attn_ctx):
    """A NaN in one row's query makes that row NaN and no other."""
    for n in (1, 3, 12):
        s = Step(40 + n, 4, 2, 128, 16, [(300, n), (20, n)], "chain")
        s.q[0, 1, 5], s.q[n, 2, 100] = np.nan, np.nan
        s.upload()
        s.call(attn_ctx)
        clean(attn_ctx)
        s.check()


def test_tree_attn_strides_of_queries_and_results(attn_ctx):
    """Head-major rows, gaps between rows and heads."""
    for n, hq in ((1, 4), (4, 8), (20, 6)):
        s = Step(50 + n, hq, 2, 128, 32, [(200, n), (77, 1)], "chain", 2)
        for how in ("head_major", "gaps"):
            if how == "head_major":
                s.qd, s.out = s.qd.contiguous(), torch.full((hq, s.rows, 128), 9.0, dtype=torch.bfloat16, device="cuda")
            else:
                wide = torch.full((s.rows, hq + 3, 136), 5.0, dtype=torch.bfloat16, device="cuda")
                wide[:, :hq, :128] = s.qd.transpose(0, 1)
                s.qd = wide[:, :hq, :128].transpose(0, 1)
                s.out = torch.full((s.rows, hq + 1, 136), 9.0, dtype=torch.bfloat16, device="cuda")[:, 1:, :128].transpose(0, 1)
            s.lse.fill_(9)
            s.call(attn_ctx)
            clean(attn_ctx)
            s.check()
            if how == "gaps":
                assert bool((s.out._base[:, :1] == 9).all()) and bool((s.out._base[:, :, 128:] == 9).all())


def test_tree_attn_without_lse_gives_the_same(attn_ctx):
    s = Step(60, 8, 2, 128, 16, [(300, 2), (9, 1)], "chain")
    s.call(attn_ctx)
    first = s.out.clone()
    s.out.fill_(9)
    attn_ctx.sp_tree_attn_q4(s.qd, s.cd, s.table_d, s.lens_d, s.start_d, s.out)
    clean(attn_ctx)
    assert torch.equal(first, s.out)


@pytest.mark.parametrize("n", [1, 5, 9])
def test_tree_attn_graph_replays_with_other_lengths(attn_ctx, n):
    """One captured graph serves steps of other lengths, tables and rows."""
    a = Step(11, 8, 2, 128, 32, [(300, n), (40, 2), (0, 1)], "tree", 6)
    a.call(attn_ctx)                                                           # workspaces exist before the capture
    clean(attn_ctx)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.call(attn_ctx)
    a.blank()
    g.replay()
    clean(attn_ctx)
    a.check()
    b = Step(12, 8, 2, 128, 32, [(310, n), (0, 4), (15, 5)], "tree", 0)
    assert b.rows == a.rows and b.cache.shape[0] <= a.cache.shape[0] and b.table.shape == a.table.shape
    if b.bits.shape != a.bits.shape:
        pytest.fail("the two steps' masks differ in words")
    for name in ("qd", "table_d", "lens_d", "start_d", "bits_d"):
        getattr(a, name).copy_(getattr(b, name))
    a.cd[: b.cache.shape[0]].copy_(b.cd)
    a.blank()
    g.replay()
    clean(attn_ctx)
    b.out, b.lse = a.out, a.lse
    b.check()


def test_tree_attn_first_call_inside_a_capture(binding):  # noqa: F811
    """Without a workspace the call is refused and the capture stays good; with sp_ctx_reserve_decode it is not."""
    s = Step(70, 4, 2, 64, 16, [(100, 2)], "chain")
    ctx = binding.Context()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(binding.SpError) as e:
            s.call(ctx)
        s.lse.add_(0)
    assert e.value.code == binding.SP_ERR_WORKSPACE
    g.replay()
    ctx.reserve_decode()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.call(ctx)
    g.replay()
    clean(ctx)
    s.check()


def test_workspaces_are_made_while_another_stream_is_captured(binding):  # noqa: F811
    """A first call on a stream that is not being captured leaves a capture on another one as it is."""
    from tests import test_gpu_decode as bf
    a, b = Step(73, 4, 2, 64, 16, [(100, 2)], "chain"), bf.Step(74, 4, 2, 64, 16, [(100, 2)], "chain")
    c, d = binding.Context(), binding.Context()
    x = torch.zeros(4, device="cuda")
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode="relaxed"):
        x.add_(1)
        with torch.cuda.stream(other):
            a.call(c)
            b.call(d)
        x.add_(1)
    g.replay()
    torch.cuda.synchronize()
    assert x.tolist() == [2.0] * 4
    for ctx, step in ((c, a), (d, b)):
        clean(ctx)
        step.check()


def test_tree_attn_beside_the_bf16_one_in_one_workspace(binding):  # noqa: F811
    """The two forms take turns with one context's workspace, in a graph that holds both."""
    from tests import test_gpu_decode as bf
    ctx = binding.Context()
    a, b = Step(71, 8, 2, 128, 32, [(3000, 2), (40, 1)], "chain"), bf.Step(72, 8, 2, 128, 32, [(2500, 9), (40, 3)], "tree")
    a.call(ctx)
    b.call(ctx)
    clean(ctx)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):
            a.call(ctx)
            b.call(ctx)
    for x in (a, b):
        x.out.fill_(9)
        x.lse.fill_(9)
    g.replay()
    clean(ctx)
    a.check()
    b.check()


def test_tree_attn_contexts_on_two_streams(binding):  # noqa: F811
    streams = [torch.cuda.Stream() for _ in range(2)]
    steps = [Step(80 + i, 8, 2, 128, 16, [(4000 + 100 * i, 1 + 3 * i), (90, 1)], "chain") for i in range(2)]
    ctxs = [binding.Context() for _ in range(2)]
    for c in ctxs:
        c.reserve_decode()
    torch.cuda.synchronize()
    for _ in range(20):
        for s, c, st in zip(steps, ctxs, streams):
            with torch.cuda.stream(st):
                s.blank()
                s.call(c)
    for s, c in zip(steps, ctxs):
        clean(c)
        s.check()


def test_tree_attn_as_many_requests_as_allowed(attn_ctx):
    s = Step(90, 2, 1, 64, 16, [(i % 40, 1 if i % 7 else 0) for i in range(4096)], "chain", 3)
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()


@pytest.mark.parametrize("n", [1, 3, 12])
def test_tree_attn_page_outside_the_cache_is_reported_not_followed(binding, n):  # noqa: F811
    """Page ids are checked against the cache before they are used; the other requests come out as ever."""
    for kernel in ("simt", "tc"):
        ctx = binding.Context(kernel=kernel)
        for bad in (10 ** 6, -1):
            s = Step(31, 4, 2, 64, 16, [(100, n), (50, 3)], "chain")
            s.table_d[0, 2] = bad
            s.call(ctx)
            torch.cuda.synchronize()
            assert ctx.status() == (binding.SP_ERR_RANGE, 71) and ctx.status() == (0, 0)
            s.check(skip=(0,))
        s = Step(32, 4, 2, 64, 16, [(100, n)], "chain")
        s.lens_d.fill_(10 ** 6)                                                # longer than the table row
        s.table_d.fill_(0)
        s.call(ctx)
        torch.cuda.synchronize()
        assert ctx.status() == (binding.SP_ERR_RANGE, 71)


def test_offsets_past_32_bits(binding):  # noqa: F811
    """A cache of more than 2^32 bytes, the pages in use at its end."""
    hkv, d, page = 8, 128, 128
    per = hkv * q4.page_bytes(page, d)
    total = 2 ** 32 // per + 60
    cache = torch.zeros(total, hkv, q4.page_bytes(page, d), dtype=torch.uint8, device="cuda")
    for n in (1, 4, 9):
        s = Step(21, 16, hkv, d, page, [(1500, n), (200, 1)], "tree")
        m = s.cache.shape[0]
        cache[-m:] = s.cd
        s.cd = cache
        s.table_d += (s.table_d != 2 ** 31 - 1) * (total - m)
        for kernel in ("tc", "simt"):
            ctx = binding.Context(kernel=kernel)
            s.blank()
            s.call(ctx)
            clean(ctx)
            s.check()
    slot = (total - 1) * page + 77
    x = torch.randn(1, 16 + 2 * hkv, d, device="cuda").to(torch.bfloat16)
    q, kk, vv = (y.transpose(0, 1) for y in x.split([16, hkv, hkv], 1))
    ctx.sp_qk_norm_rope_q4(q, kk, vv, i32([0]), torch.zeros(8, dtype=torch.float64), torch.empty_like(q), cache, i32([slot]))
    lens = i32([0])
    ctx.sp_cache_keep_q4(cache, i32([[total - 1]]), i32([70]), i32([[7]]), i32([1]), lens, d)
    ko, vo = (torch.empty(hkv, 71, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.sp_cache_read_q4(cache, i32([[total - 1]]), lens, i32([0, 71]), ko, vo)
    clean(ctx)
    same_codes(host(ko[:, 70]), host(kk[:, 0]), 0)
    same_codes(host(vo[:, 70]), host(vv[:, 0]), 0)
    assert lens.tolist() == [71]


# ---------------------------------------------------------------- reading and compaction

@pytest.mark.parametrize("d,hkv,page,reqs,pad,gap,major", [
    (128, 1, 16, [(1, 1)], 0, 0, True), (64, 8, 64, [(5, 5), (0, 0), (130, 130), (17, 3)], 4, 16, False), (128, 8, 16, [(100, 100), (33, 1), (16, 16), (15, 15)], 0, 0, True),
    (128, 3, 256, [(700, 700), (256, 255)], 1, 32, False), (64, 2, 128, [(3000, 2999)], 0, 0, True), (128, 2, 32, [(i % 50, i % 50) for i in range(300)], 7, 0, True),
    (64, 1, 16, [(1, 0)] * 4096, 2, 0, True)])
def test_read(binding, d, hkv, page, reqs, pad, gap, major):  # noqa: F811
    """Every byte pattern, as bf16 exactly; the last n tokens; rows behind the last request stay."""
    rng = np.random.default_rng(d + hkv + page)
    need = [-(-t // page) for t, _ in reqs]
    total = sum(need) + 1
    cache = rng.integers(0, 256, (total, hkv, q4.page_bytes(page, d)), dtype=np.uint8)
    order, at = rng.permutation(total), 0
    table = np.full((len(reqs), max(max(need), 1)), -1)
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    rows = sum(n for _, n in reqs) + pad
    make = (lambda: torch.full((hkv, rows, d), 9.0, dtype=torch.bfloat16, device="cuda")) if major else (
        lambda: torch.full((rows, hkv, d + 8), 9.0, dtype=torch.bfloat16, device="cuda")[:, :, :d].transpose(0, 1))
    ko, vo = make(), make()
    ctx = binding.Context()
    ctx.sp_cache_read_q4(u8(cache, gap), i32(table), i32([t for t, _ in reqs]), i32(np.cumsum([0] + [n for _, n in reqs])), ko, vo)
    clean(ctx)
    values = q4.unpack(cache, page, d)
    for got, c in zip((host(ko), host(vo)), values):
        start = 0
        for b, (t, n) in enumerate(reqs):
            p = np.arange(t - n, t)
            assert np.array_equal(got[:, start:start + n], c[table[b][p // page], :, p % page].transpose(1, 0, 2) if n else got[:, start:start])
            start += n
        assert np.all(got[:, start:] == 9)
    if not major:
        assert bool((ko._base[:, :, d:] == 9).all())


def test_read_outside_the_table_is_reported_not_followed(binding):  # noqa: F811
    ctx = binding.Context()
    cache = torch.randint(0, 256, (4, 2, q4.page_bytes(16, 64)), dtype=torch.uint8, device="cuda")
    values = q4.unpack(cache.cpu().numpy(), 16, 64)
    for table, lens, start, fine in (([[0, 9], [1, 2]], [20, 20], [0, 20, 40], range(20, 40)), ([[0, -1], [1, 2]], [20, 20], [0, 20, 40], range(20, 40)),
                                     ([[0, 3], [1, 2]], [40, 20], [0, 20, 40], range(20, 40)), ([[0, 3], [1, 2]], [5, 20], [0, 20, 40], range(20, 40))):
        ko, vo = (torch.full((2, 40, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ctx.sp_cache_read_q4(cache, i32(table), i32(lens), i32(start), ko, vo)
        torch.cuda.synchronize()
        assert ctx.status() == (binding.SP_ERR_RANGE, 86) and ctx.status() == (0, 0)
        want = values[0][[1, 2]].transpose(1, 0, 2, 3).reshape(2, 32, 64)[:, :20]
        assert np.array_equal(host(ko)[:, 20:], want)


@pytest.mark.parametrize("hkv,d,page,n,most", [(1, 64, 16, 1, 1), (8, 128, 16, 9, 12), (4, 128, 64, 40, 64), (2, 64, 256, 5, 256), (3, 128, 32, 7, 70)])
def test_keep(binding, hkv, d, page, n, most):  # noqa: F811
    rng = random.Random(n)
    past = [rng.choice([0, 1, page - 1, page, 3 * page + 5]) for _ in range(n)]
    new = [rng.randint(1, most) for _ in range(n)]
    new[0] = most
    counts = [rng.choice([0, 1, m, rng.randint(0, m)]) for m in new]
    counts[0] = max(1, most - 1)
    kept = [sorted(rng.sample(range(m), c)) for m, c in zip(new, counts)]
    width = -(-(max(past) + most) // page)
    total = n * width
    ids = list(range(total))
    rng.shuffle(ids)
    table = [ids[b * width:(b + 1) * width] for b in range(n)]
    cache = np.random.default_rng(n).integers(0, 256, (total, hkv, q4.page_bytes(page, d)), dtype=np.uint8)
    cd, lens = u8(cache, 16), i32([-7] * n)
    ctx = binding.Context()
    ctx.sp_cache_keep_q4(cd, i32(table), i32(past), i32([k + [-9] * (most - len(k)) for k in kept]), i32(counts), lens, d)
    clean(ctx)
    want = cache.copy()
    for b in range(n):
        for i, j in enumerate(kept[b]):
            src, dst = past[b] + j, past[b] + i
            for head in range(hkv):
                frm, to = (x[table[b][p // page], head, p % page // 16 * 17 * d:][:17 * d] for x, p in ((cache, src), (want, dst)))
                # an element's byte for the destination is the source's byte of the same element
                for which in range(4):
                    to[q4.places(dst % 16, d)[which]] = frm[q4.places(src % 16, d)[which]]
    assert np.array_equal(cd.cpu().numpy(), want) and lens.tolist() == [p + c for p, c in zip(past, counts)]


def test_keep_outside_the_table_is_reported_not_followed(binding):  # noqa: F811
    ctx = binding.Context()
    cache = torch.randint(0, 256, (3, 1, q4.page_bytes(16, 64)), dtype=torch.uint8, device="cuda")
    before = cache.clone()
    lens = i32([0, 0])
    for table, kept in (([[0, 7], [1, 2]], [[15, 0], [0, 1]]), ([[0, -1], [1, 2]], [[15, 0], [0, 1]]), ([[0, 1], [1, 2]], [[40, 0], [0, 1]]), ([[0, 1], [1, 2]], [[-1, 0], [0, 1]])):
        ctx.sp_cache_keep_q4(cache, i32(table), i32([10, 0]), i32(kept), i32([1, 2]), lens, 64)
        torch.cuda.synchronize()
        assert ctx.status() == (binding.SP_ERR_RANGE, 81) and ctx.status() == (0, 0)
        assert torch.equal(cache, before) and lens.tolist() == [11, 2]


def test_a_step_without_requests_is_no_work(binding):  # noqa: F811
    ctx = binding.Context()
    none = i32([]).view(0)
    cache = torch.zeros(2, 2, q4.page_bytes(16, 64), dtype=torch.uint8, device="cuda")
    for rows in (0, 3):
        q, out = (torch.full((4, rows, 64), 2.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ctx.sp_tree_attn_q4(q, cache, none.view(0, 4), none, i32([0]), out, lse_out=torch.ones(4, rows, device="cuda"))
        ctx.sp_cache_read_q4(cache, none.view(0, 4), none, i32([0]), q[:2], out[:2])
        clean(ctx)
        assert bool((out == 2).all())
    ctx.sp_cache_keep_q4(cache, none.view(0, 4), none, none.view(0, 3), none, none, 64)
    ctx.sp_cache_keep_q4(cache, i32([[0]]), i32([3]), i32([]).view(1, 0), i32([0]), none.new_zeros(1), 64)
    clean(ctx)


def test_wrong_shapes_are_named(binding):  # noqa: F811
    s = Step(1, 4, 2, 64, 16, [(5, 2)])
    ctx = binding.Context()
    with pytest.raises(ValueError, match="cache: expected \\[pages, heads"):
        ctx.sp_tree_attn_q4(s.qd, s.cd[0], s.table_d, s.lens_d, s.start_d, s.out)
    with pytest.raises(ValueError, match="cache: pages of 1088 bytes do not hold heads of 128 elements"):
        ctx.sp_cache_keep_q4(s.cd, s.table_d, s.lens_d, i32([[0]]), i32([1]), s.lens_d.clone(), 128)
    with pytest.raises(ValueError, match="tree_mask: expected at least one word"):
        ctx.sp_tree_attn_q4(s.qd, s.cd, s.table_d, s.lens_d, s.start_d, s.out, tree_mask=torch.zeros(2, 0, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="seq_lens"):
        ctx.sp_cache_read_q4(s.cd, s.table_d, s.lens_d.float(), s.start_d, s.qd[:2], s.out[:2])
    with pytest.raises(binding.SpError, match="-1"):
        ctx.sp_tree_attn_q4(s.qd, s.cd, s.table_d, s.lens_d, s.start_d, s.qd)


# ---------------------------------------------------------------- a run of them together

def test_prompt_then_tree_steps(binding):  # noqa: F811
    """A prompt into the cache and through the prefill call, two steps of drafted trees with compaction between them, and the
    cached prefix read back: every result against float64 on the tokens that were kept."""
    hq, hkv, d, page, prompt = 8, 2, 128, 32, 256
    rng = random.Random(1)
    g = torch.Generator().manual_seed(2)
    ctx = binding.Context()
    width = 14
    free = list(range(40))
    rng.shuffle(free)
    cache = torch.zeros(40, hkv, binding.page_bytes(page, d), dtype=torch.uint8, device="cuda")
    table, lens, start = i32([[-1] * width]), i32([0]), i32([0, 0])
    freq = 1e4 ** (-np.arange(64) / 64.0)
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16) for _ in range(2))
    K, V = np.zeros((hkv, 0, d)), np.zeros((hkv, 0, d))
    past = i32([0])

    def step(n, parents):
        nonlocal free
        words = -(-n // 32)
        pos, slots, info = i32([0] * n), i32([-1] * n), i32([0] * 4)
        bits = torch.zeros(n, words, dtype=torch.int32, device="cuda") if parents else None
        ctx.sp_page_tables(past, i32([n]), page, i32(free), table, lens, start, pos, slots, info, parents=i32(parents) if parents else None, tree_mask=bits)
        free = free[info.tolist()[1]:]
        x = torch.randn(n, hq + 2 * hkv, d, generator=g).to(torch.bfloat16).cuda()
        q, k, v = (y.transpose(0, 1) for y in x.split([hq, hkv, hkv], 1))
        q_out = torch.empty(hq, n, d, dtype=torch.bfloat16, device="cuda")
        k_out, v_out = (torch.empty(hkv, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ctx.sp_qk_norm_rope_q4(q, k, v, pos, torch.tensor(freq), q_out, cache, slots, k_out, v_out, wq.cuda(), wk.cuda())
        at = pos.cpu().numpy()
        k64, _ = ref.norm_rope(host(k), host(wk), 1e-6, freq, False, at)
        coded = [q4.values(*q4.quantise(y)[:2]) for y in (k64, host(v))]
        return q_out, k_out, v_out, coded, bits

    q_out, k_out, v_out, (nk, nv), _ = step(prompt, None)
    out = torch.empty_like(q_out)
    ctx.sp_prefill_attn(q_out, k_out, v_out, [0] * hq, [0], 0.9, 128, out)
    K, V = nk, nv
    past = i32([prompt])
    for n in (20, 7):
        parents = tree(rng, n)
        q_out, _, _, (nk, nv), bits = step(n, parents)
        out, lse = torch.empty_like(q_out), torch.empty(hq, n, device="cuda")
        ctx.sp_tree_attn_q4(q_out, cache, table, lens, start, out, tree_mask=bits, lse_out=lse)
        paths = []
        for j in range(n):
            paths.append((paths[parents[j]] if parents[j] >= 0 else []) + [j])
        seen = np.array([[x < K.shape[1] or x - K.shape[1] in paths[j] for x in range(K.shape[1] + n)] for j in range(n)])
        for h in range(hq):
            want, want_lse, tol = ref.attention(host(q_out)[h], np.concatenate([K, nk], 1)[h // 4], np.concatenate([V, nv], 1)[h // 4], seen)
            assert np.all(np.abs(host(out)[h] - want) <= tol) and np.all(np.abs(lse[h].cpu().numpy() - want_lse) <= 2.0 ** -11 + 2.0 ** -20 * np.abs(want_lse))
        kept = max(paths, key=len)
        kept_lens = i32([0])
        ctx.sp_cache_keep_q4(cache, table, past, i32([kept]), i32([len(kept)]), kept_lens, d)
        K, V = np.concatenate([K, nk[:, kept]], 1), np.concatenate([V, nv[:, kept]], 1)
        past = kept_lens
    total = K.shape[1]
    assert past.tolist() == [total]
    ko, vo = (torch.empty(hkv, total, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.sp_cache_read_q4(cache, table, past, i32([0, total]), ko, vo)
    clean(ctx)
    assert np.array_equal(host(ko), K) and np.array_equal(host(vo), V)
