"""The decode-side operators on the GPU against plain float64 statements: small sizes at which they can go wrong."""
import random

import numpy as np
import pytest
import torch

from tests import _decode_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2505_19578_b200 import binding as b, build
    build.build()
    return b


@pytest.fixture(scope="module", params=["tc", "simt"])
def attn_ctx(binding, request):
    return binding.Context(kernel=request.param)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.float32).to(torch.bfloat16).cuda()


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def clean(ctx):
    torch.cuda.synchronize()
    assert ctx.status() == (0, 0)


# ---------------------------------------------------------------- page tables

def tree(rng, n):
    return [max(-1, j - 1 - int(rng.random() * rng.random() * 6)) for j in range(n)]


def run_tables(binding, ctx, past, new, page, free, table, rows, parents=None, words=0):
    n = len(past)
    t, lens, start = i32(table), i32([-7] * n), i32([-7] * (n + 1))
    pos, slots, info = i32([-7] * rows), i32([-9] * rows), i32([-7] * 4)
    bits = torch.full((rows, words), -5, dtype=torch.int32, device="cuda") if parents is not None else None
    ctx.sp_page_tables(i32(past), i32(new), page, i32(free), t, lens, start, pos, slots, info,
                       parents=None if parents is None else i32(parents), tree_mask=bits)
    clean(ctx)
    return t, lens, start, pos, slots, bits, info


def same_tables(got, want, rows, words):
    t, lens, start, pos, slots, bits, info = got
    wt, wl, ws, wp, wsl, wb, wi = want
    assert t.tolist() == wt.tolist() and lens.tolist() == wl and start.tolist() == ws
    assert pos.tolist() == [-7 if x is None else x for x in wp]
    assert slots.tolist() == [-9 if x is None else x for x in wsl]
    if bits is not None:
        assert [[w & 0xFFFFFFFF for w in r] for r in bits.tolist()] == [[0xFFFFFFFB] * words if r is None else r for r in wb]
    assert info.tolist() == wi


@pytest.mark.parametrize("n,page,top,new,words,spare", [
    (1, 16, 0, 1, 0, 0), (1, 64, 1000, 1, 0, 3), (7, 16, 40, 5, 0, 2), (33, 32, 300, 9, 1, 5), (64, 128, 5000, 64, 2, 0), (300, 16, 200, 40, 2, 17),
    (1000, 256, 3000, 3, 1, 1), (4096, 16, 50, 2, 0, 1), (3, 16, 100, 256, 8, 9), (2, 64, 0, 5000, 0, 4)])
def test_page_tables(binding, n, page, top, new, words, spare):
    rng = random.Random(n * 31 + page)
    past = [rng.choice([0, 1, page - 1, page, page + 1, top, rng.randint(0, top)]) for _ in range(n)]
    past = [min(p, top) for p in past]
    fresh = [rng.choice([0, 1, new, rng.randint(0, new)]) for _ in range(n)]
    fresh[0] = max(fresh[0], 1)
    width = -(-(top + new) // page) + 1
    ids = list(range(n * width))
    rng.shuffle(ids)
    table = [[ids.pop() if c * page < p else -3 for c in range(width)] for p in past]
    rows = sum(fresh) + spare
    parents = None
    if words:
        parents = [x for f in fresh for x in tree(rng, f)] + [12345] * spare
    args = (past, fresh, page, ids, table, rows, parents, words)
    want = ref.page_tables(*args)
    ctx = binding.Context()
    got = run_tables(binding, ctx, *args)
    same_tables(got, want, rows, words)


def test_page_tables_failures_are_counted_and_stay_in_bounds(binding):
    """Negative lengths, a row that is too short, no page left, a tree wider than its mask, bad parents, rows that do not fit."""
    ctx = binding.Context()
    past, new = [5, -4, 60, 0, 16, 2], [3, 2, 10, 40, 1, 0]
    table = [[1, -1, -1, -1], [-1] * 4, [8, 9, 10, 11], [-1] * 4, [2, -1, -1, -1], [3, -1, -1, -1]]
    parents = [-1, 0, 5, -2, 0] + [-1] * 10 + list(range(-1, 39)) + [-1]
    for free, rows in (([20, 21, 22, 23], 56), ([20, 21], 56), ([20, 21], 30), ([], 56)):
        p = (parents + [-1] * 60)[:rows]
        args = (past, new, 16, free, table, rows, p, 1)
        same_tables(run_tables(binding, ctx, *args), ref.page_tables(*args), rows, 1)


def test_page_tables_again_and_empty_steps(binding):
    """Called twice with the same lengths: the same values.  A step in which nobody gets anything: no rows."""
    ctx = binding.Context()
    table, lens, start, pos, slots, _, info = run_tables(binding, ctx, [17, 0], [3, 2], 16, [5, 6], [[1, 2, -1], [-1, -1, -1]], 6)
    first = [x.clone() for x in (table, lens, start, pos, slots, info)]
    ctx.sp_page_tables(i32([17, 0]), i32([3, 2]), 16, i32([5, 6]), table, lens, start, pos, slots, info)
    clean(ctx)
    assert all(torch.equal(a, b) for a, b in zip(first, (table, lens, start, pos, slots, info)))
    table, lens, start, pos, slots, _, info = run_tables(binding, ctx, [17, 0], [0, 0], 16, [], [[1, 2], [-1, -1]], 2)
    assert start.tolist() == [0, 0, 0] and slots.tolist() == [-9, -9] and info.tolist() == [0, 0, 0, 17] and lens.tolist() == [17, 0]


# ---------------------------------------------------------------- norm and rotation

def rope_case(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, major, seed=0, scale=1.0):
    rng = np.random.default_rng(seed)
    qkv = ref.bf16_values(rng, rows, hq + 2 * hkv, d, scale=scale)
    weights = [ref.bf16_values(rng, d) if norm else None for _ in range(2)]
    freq = 5e5 ** (-np.arange(n_freq) * 2.0 / max(1, 2 * n_freq))
    pos = rng.integers(0, 131072, rows)
    pos[: min(rows, 3)] = [0, 2 ** 31 - 1, 1][: min(rows, 3)]
    t = dev(qkv)
    q, k, v = (x.transpose(0, 1) for x in t.split([hq, hkv, hkv], 1))
    make = (lambda h: torch.full((h, rows, d), 7.0, dtype=torch.bfloat16, device="cuda")) if major else (
        lambda h: torch.full((rows, h, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1))
    q_out, k_out, v_out = make(hq), *((make(hkv), make(hkv)) if outs else (None, None))
    kc = vc = slots = None
    if page:
        pages = -(-rows // page) + 2
        kc, vc = (torch.full((pages, hkv, page, d), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        slots = rng.permutation(pages * page)[:rows]
        slots[rng.random(rows) < 0.2] = -1
    ctx = binding.Context()
    ctx.sp_qk_norm_rope(q, k, v, i32(pos), torch.tensor(freq, dtype=torch.float64), q_out, k_out, v_out, kc, vc,
                        None if slots is None else i32(slots), None if not norm else dev(weights[0]), None if not norm else dev(weights[1]), 1e-6, interleaved)
    clean(ctx)
    x = qkv.transpose(1, 0, 2)
    wq, eq = ref.norm_rope(x[:hq], weights[0], 1e-6, freq, interleaved, pos)
    wk, ek = ref.norm_rope(x[hq:hq + hkv], weights[1], 1e-6, freq, interleaved, pos)
    wv = x[hq + hkv:]
    eq, ek = eq + ref.EPS_BF16 * np.abs(wq), ek + ref.EPS_BF16 * np.abs(wk)
    assert np.all(np.abs(host(q_out) - wq) <= eq)
    if outs:
        assert np.all(np.abs(host(k_out) - wk) <= ek) and np.array_equal(host(v_out), wv)
    if page:
        fk, fv = (host(c).transpose(0, 2, 1, 3).reshape(-1, hkv, d) for c in (kc, vc))
        used = np.zeros(len(fk), dtype=bool)
        for r, s in enumerate(slots):
            if s >= 0:
                used[s] = True
                assert np.all(np.abs(fk[s] - wk[:, r]) <= ek[:, r]) and np.array_equal(fv[s], wv[:, r])
        assert np.all(fk[~used] == 3) and np.all(fv[~used] == 3)                # nothing else was written


@pytest.mark.parametrize("hq,hkv,d,rows,n_freq,interleaved,norm,outs,page,major", [
    (32, 8, 128, 1, 64, False, False, False, 64, False), (32, 8, 128, 1, 64, False, True, True, 0, True), (28, 4, 128, 37, 64, False, True, True, 16, True),
    (8, 8, 64, 129, 32, False, True, False, 32, False), (8, 8, 64, 5, 32, True, True, True, 16, False), (7, 1, 128, 3, 32, False, False, True, 0, False),
    (5, 5, 64, 2, 8, True, False, True, 256, True), (16, 2, 128, 1000, 64, True, True, True, 128, True), (3, 1, 64, 70, 16, False, True, True, 64, True),
    (128, 128, 128, 2, 64, False, True, True, 16, True), (1, 1, 64, 1, 0, False, True, True, 16, True), (4, 2, 128, 9, 0, False, False, True, 0, True),
    (2, 1, 128, 6000, 64, False, True, True, 16, True)])
def test_norm_rope(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, major):
    rope_case(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, major)


def test_norm_rope_of_tiny_and_huge_values(binding):
    rope_case(binding, 4, 2, 128, 11, 64, False, True, True, 16, True, seed=3, scale=2.0 ** 40)
    rope_case(binding, 4, 2, 128, 11, 64, False, True, True, 16, True, seed=4, scale=2.0 ** -12)


def test_norm_rope_in_place_and_on_another_stream(binding):
    rng = np.random.default_rng(5)
    x = ref.bf16_values(rng, 50, 12, 128)
    freq = 5e5 ** (-np.arange(64) / 64.0)
    pos = rng.integers(0, 131072, 50)
    t = dev(x)
    pos_d = i32(pos)
    q, k, v = (y.transpose(0, 1) for y in t.split([8, 2, 2], 1))
    ctx = binding.Context()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ctx.sp_qk_norm_rope(q, k, v, pos_d, torch.tensor(freq), q, k, v, stream=s)
    s.synchronize()
    clean(ctx)
    x = x.transpose(1, 0, 2)
    want, err = ref.norm_rope(x[:10], None, 0, freq, False, pos)
    assert np.all(np.abs(host(t).transpose(1, 0, 2)[:10] - want) <= err + ref.EPS_BF16 * np.abs(want))
    assert np.array_equal(host(v), x[10:])


def test_norm_rope_slot_behind_the_cache_is_reported_not_followed(binding):
    ctx = binding.Context()
    x = torch.randn(3, 4, 64, device="cuda").to(torch.bfloat16)
    kc, vc = (torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, k, v = x[:, :2].transpose(0, 1), x[:, 2:3].transpose(0, 1), x[:, 3:].transpose(0, 1)
    freq = torch.ones(0, dtype=torch.float64)
    ctx.sp_qk_norm_rope(q, k, v, i32([0, 1, 2]), freq, torch.empty_like(q), k_cache=kc, v_cache=vc, slots=i32([31, 32, 2 ** 31 - 1]))
    torch.cuda.synchronize()
    assert ctx.status() == (binding.SP_ERR_RANGE, 75) and ctx.status() == (0, 0)
    assert torch.equal(vc[1, 0, 15], x[0, 3]) and float(vc.float().abs().sum()) == float(x[0, 3].float().abs().sum())


# ---------------------------------------------------------------- attention over the cache

class Step:
    """Inputs of one call, host copies beside them."""

    def __init__(self, seed, hq, hkv, d, page, reqs, kind="chain", pad=0, layout="paged", spoil=None, scale=1.0):
        r, rng = random.Random(seed), np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.page, self.reqs = hq, hkv, d, page, reqs
        rows = sum(n for _, n in reqs) + pad
        self.rows = rows
        self.q = ref.bf16_values(rng, rows, hq, d, scale=scale)
        need = [-(-(p + n) // page) for p, n in reqs]
        width = max(max(need), 1) + 1
        total = sum(need) + 2
        order = list(range(total))
        if layout == "paged":
            r.shuffle(order)
        self.table = np.full((len(reqs), width), 2 ** 31 - 1)              # entries behind the last page are not read
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.k, self.v = ref.bf16_values(rng, total, hkv, page, d), ref.bf16_values(rng, total, hkv, page, d)
        self.bits, self.words = None, 0
        if kind != "chain":
            most = max(n for _, n in reqs)
            self.words = -(-most // 32)
            self.bits = np.zeros((rows, self.words), dtype=np.int64)
            t = 0
            for p, n in reqs:
                parents = tree(r, n)
                seen = []
                for j in range(n):
                    s = (seen[parents[j]] if parents[j] >= 0 else 0) | 1 << j
                    seen.append(s)
                    if kind == "any":                                      # any bits at all, some rows none
                        s = r.getrandbits(n) if j % 3 else 0
                    for w in range(self.words):
                        self.bits[t + j, w] = (s >> (32 * w)) & 0xFFFFFFFF
                t += n
            self.bits[t:] = 0xFFFFFFFF
        self.spoil(spoil, rng)
        if layout == "contiguous":
            # pages of one head side by side, as in [heads, seq, head_dim]
            self.kd, self.vd = (dev(x.transpose(1, 0, 2, 3)).reshape(hkv, total * page, d).unflatten(1, (total, page)).transpose(0, 1) for x in (self.k, self.v))
        elif layout == "token_major":
            self.kd, self.vd = (dev(x.transpose(0, 2, 1, 3)).transpose(1, 2) for x in (self.k, self.v))
        else:
            self.kd, self.vd = dev(self.k), dev(self.v)
        self.qd = dev(self.q).transpose(0, 1)
        self.out = torch.full((rows, hq, d), 9.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
        self.lse = torch.full((hq, rows), 9.0, device="cuda")
        self.lens_d, self.start_d = i32([p + n for p, n in reqs]), i32(np.cumsum([0] + [n for _, n in reqs]))
        self.table_d = i32(self.table)
        self.bits_d = None if self.bits is None else torch.tensor(self.bits).to(torch.int32).cuda()

    def spoil(self, what, rng):
        if what is None:
            return
        bad = {"nan": np.nan, "inf": np.inf, "-inf": -np.inf}[what]
        used = np.zeros(self.k.shape[:1] + (self.page,), dtype=bool)
        for b, (p, n) in enumerate(self.reqs):
            for x in range(p + n):
                used[self.table[b, x // self.page], x % self.page] = True
        self.k.transpose(0, 2, 1, 3)[~used] = bad
        self.v.transpose(0, 2, 1, 3)[~used] = bad
        if self.bits is not None:
            # and in drafted tokens, which only their own branch sees
            for b, (p, n) in enumerate(self.reqs):
                for x in range(1, n, 3):
                    page, off = self.table[b, (p + x) // self.page], (p + x) % self.page
                    (self.k if x % 2 else self.v)[page, :, off, x % self.d] = bad

    def call(self, ctx, **kw):
        ctx.sp_tree_attn(self.qd, self.kd, self.vd, self.table_d, self.lens_d, self.start_d, self.out, tree_mask=self.bits_d, lse_out=self.lse, **kw)

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

    def check(self):
        out, lse = host(self.out), self.lse.cpu().numpy().astype(np.float64)
        with np.errstate(all="ignore"):
            for h, rows, want, want_lse, tol in self.reference():
                got, got_lse = out[h, rows], lse[h, rows]
                fine = np.isfinite(want)
                assert np.array_equal(fine, np.isfinite(got)), (h, rows)
                assert np.all(np.isnan(want[~fine]) == np.isnan(got[~fine])) and np.all((want == got)[~fine & ~np.isnan(want)])
                far = np.abs(got - want)[fine] - tol[fine]
                assert np.all(far <= 0), (h, rows, float(far.max()), float(np.abs(got - want)[fine].max()))
                f = np.isfinite(want_lse)
                assert np.array_equal(f, np.isfinite(got_lse)) and np.array_equal(np.isnan(want_lse), np.isnan(got_lse))
                assert np.all(np.abs(got_lse - want_lse)[f] <= 2.0 ** -11 + 2.0 ** -20 * np.abs(want_lse[f]))
        end = sum(n for _, n in self.reqs)
        assert np.all(out[:, end:] == 9) and np.all(lse[:, end:] == 9)        # rows behind the last request: as they were


ATTN = [
    # hq, hkv, d, page, requests (past, new), kind, pad, layout
    (1, 1, 64, 16, [(0, 1)], "chain", 0, "paged"),
    (8, 8, 64, 64, [(2047, 1)], "chain", 0, "paged"),
    (32, 8, 128, 128, [(1, 1), (0, 1), (127, 1), (128, 1), (129, 1), (1000, 1)], "chain", 3, "paged"),
    (28, 4, 128, 16, [(5, 16), (0, 16), (300, 7), (111, 1), (112, 16)], "tree", 2, "paged"),
    (32, 8, 128, 32, [(513, 64)], "tree", 0, "paged"),
    (8, 1, 128, 64, [(70, 64), (3, 33)], "tree", 5, "contiguous"),
    (16, 4, 64, 256, [(700, 20), (0, 0), (255, 2)], "chain", 1, "token_major"),
    (4, 4, 64, 16, [(40, 100)], "any", 0, "paged"),
    (6, 2, 128, 16, [(0, 40), (0, 3), (17, 5)], "any", 4, "paged"),
    (2, 1, 128, 32, [(10, 256)], "tree", 0, "paged"),
    (4, 2, 128, 128, [(600, 300)], "chain", 0, "contiguous"),
    (16, 1, 64, 16, [(9, 9)] * 40, "tree", 0, "paged"),
    (8, 8, 128, 64, [(3, 1)] * 150 + [(2000, 1)] + [(0, 2)] * 5, "chain", 0, "paged"),
    (128, 128, 64, 16, [(50, 2)], "chain", 0, "paged"),
    (128, 1, 128, 16, [(50, 3)], "tree", 0, "paged"),
    (2, 2, 64, 16, [(0, 0), (0, 0), (0, 1), (0, 0)], "chain", 0, "paged"),
    # at most eight rows per request and key head
    (8, 8, 128, 16, [(0, 8), (3, 1), (200, 5), (0, 0), (1000, 8), (121, 7)], "tree", 1, "paged"),
    (16, 8, 128, 64, [(0, 4), (300, 3), (127, 1), (128, 2), (0, 1)], "any", 3, "contiguous"),
    (14, 2, 128, 256, [(5000, 1), (7, 1), (0, 1), (511, 1), (512, 1)], "chain", 0, "token_major"),
    (8, 1, 128, 32, [(9, 1)] * 200 + [(1900, 1)], "chain", 0, "paged"),
]


@pytest.mark.parametrize("case", ATTN, ids=[str(i) for i in range(len(ATTN))])
def test_tree_attn(attn_ctx, case):
    hq, hkv, d, page, reqs, kind, pad, layout = case
    s = Step(len(reqs) + hq, hq, hkv, d, page, reqs, kind, pad, layout)
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()
    first = s.out.clone(), s.lse.clone()
    s.call(attn_ctx)                                                          # the same bits again
    clean(attn_ctx)
    assert torch.equal(first[0].view(torch.int16), s.out.view(torch.int16)) and torch.equal(first[1], s.lse)


@pytest.mark.parametrize("spoil", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("d,page,hq,reqs", [(64, 16, 8, [(130, 40), (0, 5), (1, 70), (127, 1)]), (128, 64, 8, [(130, 40), (0, 5), (1, 70), (127, 1)]),
                                            (128, 16, 4, [(130, 4), (0, 3), (1, 4), (127, 1), (700, 4)]), (64, 32, 4, [(130, 20), (0, 3), (600, 31)])],
                         ids=["64-16", "128-64", "128-16-few", "64-32"])
def test_tree_attn_masked_and_unused_places_hold_anything(attn_ctx, spoil, d, page, hq, reqs):
    s = Step(7, hq, 2, d, page, reqs, "tree", 2, "paged", spoil)
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()


@pytest.mark.parametrize("reqs", [[(200, 3), (77, 10)], [(900, 3), (77, 4), (2000, 1)]], ids=["many rows", "few rows"])
def test_tree_attn_large_logits(attn_ctx, reqs):
    """Logits of several hundred, whose running maximum climbs from tile to tile: one key takes all."""
    s = Step(3, 4, 2, 128, 32, reqs, "tree", 0, "paged", scale=64.0)
    for b, (p, n) in enumerate(reqs):                                          # keys that get longer along the sequence
        for x in range(p + n):
            s.k[s.table[b, x // 32], :, x % 32] *= 2.0 ** -(4 - 4 * x // (p + n))
    s.kd = dev(s.k)
    s.call(attn_ctx)
    clean(attn_ctx)
    out = host(s.out)
    for h, rows, want, want_lse, tol in s.reference():
        # logits of 500 are off by d 2^-24 sum |q k| / sqrt(d) < 2^-17 * 64 * 100 / 11 nats at most
        assert np.all(np.abs(out[h, rows] - want) <= tol + 0.01 * np.abs(want).max())


def test_tree_attn_lengths_shorter_than_the_new_tokens(attn_ctx):
    """seq_lens below the number of rows: the first rows see nothing and come out as zeros."""
    s = Step(5, 4, 2, 64, 16, [(0, 6)], "chain")
    s.lens_d.fill_(4)
    s.call(attn_ctx)
    clean(attn_ctx)
    out, lse = host(s.out), s.lse.cpu().numpy()
    k, v = (c[s.table[0, :1]].transpose(1, 0, 2, 3).reshape(2, -1, 64)[:, :4] for c in (s.k, s.v))
    seen = np.array([[x + 2 <= j for x in range(4)] for j in range(6)])        # past = 4 - 6: key x is new token x + 2
    for h in range(4):
        want, want_lse, tol = ref.attention(s.q[:, h], k[h // 2], v[h // 2], seen)
        assert np.all(np.abs(out[h] - want) <= tol) and np.all(out[h, :2] == 0) and np.all(np.isneginf(lse[h, :2]))
    s.lens_d.fill_(0)
    s.call(attn_ctx)
    clean(attn_ctx)
    assert np.all(host(s.out) == 0) and bool(torch.isneginf(s.lse).all())


def test_tree_attn_graph_replays_with_other_lengths(attn_ctx):
    """One captured graph serves steps of other lengths, tables and rows; run on a stream of its own."""
    a = Step(11, 8, 2, 128, 32, [(300, 5), (40, 2), (0, 1)], "tree", 6)
    a.call(attn_ctx)                                                           # workspaces exist before the capture
    clean(attn_ctx)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.call(attn_ctx)
    a.out.fill_(9)
    a.lse.fill_(9)
    g.replay()
    clean(attn_ctx)
    a.check()
    b = Step(12, 8, 2, 128, 32, [(310, 5), (0, 4), (15, 5)], "tree", 0)
    assert b.rows == a.rows and b.k.shape[0] <= a.k.shape[0] and b.table.shape == a.table.shape
    for name in ("qd", "table_d", "lens_d", "start_d", "bits_d"):
        getattr(a, name).copy_(getattr(b, name))
    a.kd[: b.k.shape[0]].copy_(b.kd)
    a.vd[: b.k.shape[0]].copy_(b.vd)
    a.out.fill_(9)
    a.lse.fill_(9)
    g.replay()
    clean(attn_ctx)
    b.out, b.lse = a.out, a.lse
    b.check()


def test_tree_attn_offsets_past_32_bits(binding):
    """A cache of 2^32 elements, the pages in use at its end."""
    hkv, d, page = 8, 128, 128
    total = 2 ** 32 // (hkv * d * page) + 40
    s = Step(21, 16, hkv, d, page, [(1500, 4), (200, 1)], "tree")
    k, v = (torch.empty(total, hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n = s.k.shape[0]
    k[-n:], v[-n:] = s.kd, s.vd
    s.kd, s.vd = k, v
    s.table_d += (s.table_d != 2 ** 31 - 1) * (total - n)
    for kernel in ("tc", "simt"):
        ctx = binding.Context(kernel=kernel)
        s.out.fill_(9)
        s.call(ctx)
        clean(ctx)
        s.check()
    # the cache write and the compaction reach them too
    slot = (total - 1) * page + 77
    x = torch.randn(1, 16 + 2 * hkv, d, device="cuda").to(torch.bfloat16)
    q, kk, vv = (y.transpose(0, 1) for y in x.split([16, hkv, hkv], 1))
    ctx.sp_qk_norm_rope(q, kk, vv, i32([0]), torch.zeros(8, dtype=torch.float64), torch.empty_like(q), k_cache=k, v_cache=v, slots=i32([slot]))
    clean(ctx)
    assert torch.equal(v[total - 1, :, 77], vv[:, 0]) and torch.equal(k[total - 1, :, 77], kk[:, 0])
    lens = i32([0])
    ctx.sp_cache_keep(k, v, i32([[total - 1]]), i32([70]), i32([[7]]), i32([1]), lens)
    clean(ctx)
    assert torch.equal(v[total - 1, :, 70], vv[:, 0]) and torch.equal(k[total - 1, :, 70], kk[:, 0]) and lens.tolist() == [71]


def test_tree_attn_page_outside_the_cache_is_reported_not_followed(binding):
    """Page ids are checked against the cache before they are used; the other requests come out as ever."""
    for kernel in ("simt", "tc"):
        ctx = binding.Context(kernel=kernel)
        for bad in (10 ** 6, -1):
            s = Step(31, 4, 2, 64, 16, [(100, 2), (50, 3)], "chain")
            s.table_d[0, 2] = bad
            s.call(ctx)
            torch.cuda.synchronize()
            assert ctx.status() == (binding.SP_ERR_RANGE, 70) and ctx.status() == (0, 0)
            out = host(s.out)
            for h, rows, want, _, tol in s.reference():
                if rows.start > 0:
                    assert np.all(np.abs(out[h, rows] - want) <= tol)
        s = Step(32, 4, 2, 64, 16, [(100, 2)], "chain")
        s.lens_d.fill_(10 ** 6)                                                # longer than the table row
        s.table_d.fill_(0)
        s.call(ctx)
        torch.cuda.synchronize()
        assert ctx.status() == (binding.SP_ERR_RANGE, 70)


# ---------------------------------------------------------------- compaction

@pytest.mark.parametrize("hkv,d,page,n,most", [(1, 64, 16, 1, 1), (8, 128, 16, 9, 12), (4, 128, 64, 40, 64), (2, 64, 256, 5, 256)])
def test_cache_keep(binding, hkv, d, page, n, most):
    r, rng = random.Random(most), np.random.default_rng(most)
    past = [r.choice([0, 1, page - 1, page, 3 * page + 5]) for _ in range(n)]
    new = [r.randint(1, most) for _ in range(n)]
    count = [r.randint(0, x) for x in new]
    kept = [sorted(r.sample(range(x), c)) for x, c in zip(new, count)]
    need = [-(-(p + x) // page) for p, x in zip(past, new)]
    ids = list(range(sum(need) + 3))
    r.shuffle(ids)
    table = np.full((n, max(need) + 1), -1)
    for b, m in enumerate(need):
        table[b, :m] = [ids.pop() for _ in range(m)]
    total = sum(need) + 3
    k, v = ref.bf16_values(rng, total, hkv, page, d), ref.bf16_values(rng, total, hkv, page, d)
    kd, vd = dev(k), dev(v)
    lens = i32([0] * n)
    ctx = binding.Context()
    # as many as the widest request keeps; entries behind a request's own are not read
    width = max(1, max(count))
    kk = np.array([p + [10 ** 6] * (width - len(p)) for p in kept])
    ctx.sp_cache_keep(kd, vd, i32(table), i32(past), i32(kk), i32(count), lens)
    clean(ctx)
    wk, wv = k.copy(), v.copy()
    for b in range(n):
        for i, x in enumerate(kept[b]):
            s, t = past[b] + x, past[b] + i
            for w, c in ((wk, k), (wv, v)):
                w[table[b, t // page], :, t % page] = c[table[b, s // page], :, s % page]
    assert np.array_equal(host(kd), wk) and np.array_equal(host(vd), wv)
    assert lens.tolist() == [p + c for p, c in zip(past, count)]


def test_cache_keep_outside_the_table_is_reported_not_followed(binding):
    ctx = binding.Context()
    kd = torch.randn(4, 1, 16, 64, device="cuda").to(torch.bfloat16)
    before = kd.clone()
    for table, past, kept in (([[1, -1]], [10], [[7]]), ([[1, 9]], [10], [[7]]), ([[1, 2]], [10], [[1000]]), ([[1, 2]], [10], [[-1]]), ([[1, 2]], [-5], [[1]])):
        ctx.sp_cache_keep(kd, kd.clone(), i32(table), i32(past), i32(kept), i32([1]), i32([0]))
        torch.cuda.synchronize()
        assert ctx.status() == (binding.SP_ERR_RANGE, 80) and torch.equal(kd, before)


# ---------------------------------------------------------------- together

def test_prompt_then_tree_steps(binding):
    """As a server would: a prompt through norm, rotation and the prefill call (all heads dense), its keys and values in
    the cache; then three steps of drafted trees, each verified and compacted.  Every output against float64 attention
    over the sequence of accepted tokens."""
    hq, hkv, d, page, N = 8, 2, 128, 32, 256
    rng, r = np.random.default_rng(77), random.Random(77)
    freq = 5e5 ** (-np.arange(64) / 64.0)
    freq_t = torch.tensor(freq)
    wq, wk = ref.bf16_values(rng, d), ref.bf16_values(rng, d)
    ctx = binding.Context()
    n_pages, width = 20, 12
    kc, vc = (torch.full((n_pages, hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    free = i32(r.sample(range(n_pages), n_pages))
    table, past = torch.full((1, width), -1, dtype=torch.int32, device="cuda"), i32([0])

    def tables(new, parents=None, words=0):
        nonlocal free
        rows = new
        lens, start, pos, slots, info = i32([0]), i32([0, 0]), i32([0] * rows), i32([-1] * rows), i32([0] * 4)
        bits = torch.zeros(rows, words, dtype=torch.int32, device="cuda") if parents else None
        ctx.sp_page_tables(past, i32([new]), page, free, table, lens, start, pos, slots, info, parents=i32(parents) if parents else None, tree_mask=bits)
        assert info[2].item() == 0
        free = free[info[1].item():].contiguous()
        return lens, start, pos, slots, bits

    def layer(x, pos, slots, head_major):
        q, k, v = (y.transpose(0, 1) for y in dev(x).split([hq, hkv, hkv], 1))
        rows = x.shape[0]
        mk = lambda h: torch.empty(h, rows, d, dtype=torch.bfloat16, device="cuda")
        qo, ko, vo = mk(hq), mk(hkv) if head_major else None, mk(hkv) if head_major else None
        ctx.sp_qk_norm_rope(q, k, v, pos, freq_t, qo, ko, vo, kc, vc, slots, dev(wq), dev(wk))
        return qo, ko, vo

    # prompt
    x = ref.bf16_values(rng, N, hq + 2 * hkv, d)
    _, _, pos, slots, _ = tables(N)
    assert pos.tolist() == list(range(N))
    q, k, v = layer(x, pos, slots, True)
    out = torch.empty_like(q)
    ctx.sp_prefill_attn(q, k, v, [-1] * hq, [], 0.9, 128, out)
    clean(ctx)
    K, V = host(k), host(v)                                                   # accepted keys and values so far
    seen = np.tril(np.ones((N, N), dtype=bool))
    for h in (0, hq - 1):
        want, _, tol = ref.attention(host(q)[h], K[h // 4], V[h // 4], seen)
        assert np.all(np.abs(host(out)[h] - want) <= tol)
    past = i32([N])

    for step, n in enumerate((9, 40, 1)):
        parents = tree(r, n)
        words = -(-n // 32)
        lens, start, pos, slots, bits = tables(n, parents, words)
        x = ref.bf16_values(rng, n, hq + 2 * hkv, d)
        q, _, _ = layer(x, pos, slots, False)
        out, lse = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda").transpose(0, 1), torch.empty(hq, n, device="cuda")
        ctx.sp_tree_attn(q, kc, vc, table, lens, start, out, tree_mask=bits, lse_out=lse)
        clean(ctx)
        # the drafted keys as the cache has them (rotated by position = past + depth), one bf16 rounding off the plain form
        depth = []
        for j in range(n):
            depth.append(0 if parents[j] < 0 else depth[parents[j]] + 1)
        at = past.item() + np.array(depth)
        assert pos.tolist() == at.tolist()
        wkeys, err = ref.norm_rope(x[:, hq:hq + hkv].transpose(1, 0, 2), wk, 1e-6, freq, False, at)
        flat = lambda c: host(c).transpose(0, 2, 1, 3).reshape(-1, hkv, d)[slots.cpu().numpy()].transpose(1, 0, 2)
        nk, nv = flat(kc), flat(vc)
        assert np.all(np.abs(nk - wkeys) <= err + ref.EPS_BF16 * np.abs(wkeys)) and np.array_equal(nv, x[:, hq + hkv:].transpose(1, 0, 2))
        paths = []
        for j in range(n):
            paths.append((paths[parents[j]] if parents[j] >= 0 else []) + [j])
        see = np.zeros((n, K.shape[1] + n), dtype=bool)
        see[:, :K.shape[1]] = True
        for j in range(n):
            see[j, [K.shape[1] + y for y in paths[j]]] = True
        for h in range(hq):
            want, want_lse, tol = ref.attention(host(q)[h], np.concatenate([K[h // 4], nk[h // 4]]), np.concatenate([V[h // 4], nv[h // 4]]), see)
            assert np.all(np.abs(host(out)[h] - want) <= tol), step
            assert np.all(np.abs(lse[h].cpu().numpy() - want_lse) <= 2.0 ** -11 + 2.0 ** -20 * np.abs(want_lse))
        # the longest path is accepted
        path = max(paths, key=len)
        new_past = i32([0])
        ctx.sp_cache_keep(kc, vc, table, past, i32([path]), i32([len(path)]), new_past)
        clean(ctx)
        assert new_past.item() == past.item() + len(path)
        past = new_past
        K, V = np.concatenate([K, nk[:, path]], 1), np.concatenate([V, nv[:, path]], 1)
        # pages behind the accepted tokens stay in the row: the next step counts them as free again, so give them back
        used = -(-past.item() // page)
        row = table[0].tolist()
        back = [p for p in row[used:] if p >= 0]
        table[0, used:] = -1
        free = torch.cat([free, i32(back)]).contiguous()


@pytest.mark.parametrize("rise", [40.0, -40.0, 400.0], ids=["climbing", "falling", "far"])
@pytest.mark.parametrize("hq,hkv,d,reqs", [(4, 2, 128, [(700, 10), (1, 20)]), (8, 1, 64, [(513, 16), (300, 3)]), (4, 4, 128, [(260, 17)]), (2, 2, 64, [(700, 1), (200, 16)])])
def test_tree_attn_logits_far_from_the_first_tiles(attn_ctx, hq, hkv, d, reqs, rise):
    """Logits that move by `rise` from each 128 keys to the next, hundreds of nats in all."""
    s = Step(17, hq, hkv, d, 32, reqs, "tree", 0, "paged")
    # the first column carries the level
    s.q[..., 0] = 8.0
    far = 0.0
    for b, (p, n) in enumerate(reqs):
        for x in range(p + n):
            level = x // 128 * rise
            far = max(far, abs(level))
            s.k[s.table[b, x // 32], :, x % 32, 0] = float(torch.tensor(level * np.sqrt(d) / 8).to(torch.bfloat16))
    s.qd, s.kd = dev(s.q).transpose(0, 1), dev(s.k)
    s.call(attn_ctx)
    clean(attn_ctx)
    out = host(s.out)
    # an fp32 sum of d terms of which one is `far` sqrt(d): off by d 2^-23 far nats at most (truncation counted, scaled), and
    # the weights by as much of themselves
    off = d * 2.0 ** -23 * far
    for h, rows, want, want_lse, tol in s.reference():
        assert np.all(np.abs(out[h, rows] - want) <= tol + 2 * off * np.abs(s.v).max())


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
@pytest.mark.parametrize("n", [16, 17, 128, 129, 256, 257])
def test_tree_attn_row_counts_at_the_modes_edges(attn_ctx, n, d, page):
    """One query head per key head: n rows of a long and of a short request, the runs cut across both."""
    s = Step(n, 2, 2, d, page, [(1500, n), (0, min(n, 5)), (129, 1)], "tree" if n <= 256 else "chain", 1, "paged")
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()


def test_tree_attn_first_call_inside_a_capture(binding):
    """The workspace cannot be allocated there: an error, nothing enqueued; with the workspace reserved the call is captured."""
    ctx = binding.Context()
    s = Step(3, 4, 2, 64, 16, [(40, 3)])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(binding.SpError) as e:
            s.call(ctx)
        s.lse.add_(0)
    assert e.value.code == -3 and bool((s.out == 9).all())
    ctx.reserve_decode()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.call(ctx)
    assert bool((s.out == 9).all())
    g.replay()
    clean(ctx)
    s.check()


def test_tree_attn_contexts_on_two_streams(binding):
    """Two contexts at once, several calls each, one after the other on their streams."""
    steps = [Step(21, 8, 2, 128, 32, [(700, 9), (3, 1)], "tree"), Step(22, 4, 4, 64, 16, [(300, 1)] * 40)]
    ctxs, streams = [binding.Context() for _ in steps], [torch.cuda.Stream() for _ in steps]
    for c in ctxs:
        c.reserve_decode()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, c, st in zip(steps, ctxs, streams):
            with torch.cuda.stream(st):
                s.out.fill_(9)
                s.lse.fill_(9)
                s.call(c)
    for s, c in zip(steps, ctxs):
        clean(c)
        s.check()


def test_tree_attn_graph_replays_across_the_modes(attn_ctx):
    """One captured graph, whose replays have a few, a hundred and several hundred rows in a request."""
    a = Step(31, 8, 2, 64, 16, [(300, 64), (90, 1)], "tree", 0)
    a.call(attn_ctx)
    clean(attn_ctx)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.call(attn_ctx)
    for seed, reqs in ((32, [(310, 3), (80, 2)]), (33, [(250, 20), (70, 30)]), (34, [(0, 1), (0, 64)]), (35, [(300, 62), (5, 2)])):
        pad = a.rows - sum(n for _, n in reqs)
        b = Step(seed, 8, 2, 64, 16, reqs, "tree", pad)
        assert b.rows == a.rows and b.k.shape[0] <= a.k.shape[0]
        a.bits_d.fill_(-1)
        a.bits_d[:, : b.words].copy_(b.bits_d)
        a.bits_d[:, b.words:].fill_(0)
        a.table_d.fill_(2 ** 31 - 1)
        a.table_d[:, : b.table.shape[1]].copy_(b.table_d[:, : a.table.shape[1]])
        for name in ("qd", "lens_d", "start_d"):
            getattr(a, name).copy_(getattr(b, name))
        a.kd[: b.k.shape[0]].copy_(b.kd)
        a.vd[: b.k.shape[0]].copy_(b.vd)
        a.out.fill_(9)
        a.lse.fill_(9)
        g.replay()
        clean(attn_ctx)
        b.out, b.lse = a.out, a.lse
        b.check()


def test_tree_attn_as_many_requests_as_allowed(attn_ctx):
    """4096 requests, most of one token, some of none and some empty."""
    r = random.Random(5)
    reqs = [(r.choice([0, 1, 15, 16, 40]), r.choice([1, 1, 1, 0])) for _ in range(4096)]
    s = Step(41, 2, 1, 64, 16, reqs, "chain", 3)
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()


@pytest.mark.parametrize("n", [1, 20, 70])
def test_tree_attn_a_bad_row_stays_its_own(attn_ctx, n):
    """NaN in one request's queries, and infinities in another's: no other row is touched."""
    s = Step(51, 4, 2, 128, 32, [(200, n), (300, n), (5, n)], "tree", 0)
    s.call(attn_ctx)
    clean(attn_ctx)
    want = s.out.clone()
    s.qd[:, n // 2, 3] = float("nan")
    s.qd[:, n + n // 2, 5] = float("inf")
    s.out.fill_(9)
    s.call(attn_ctx)
    clean(attn_ctx)
    rows = [x for x in range(3 * n) if x not in (n // 2, n + n // 2)]
    # the same but for the reference that a row is given (exact), or for the walk with which a run was done: twice the bound of
    # a bf16 result
    assert torch.isfinite(s.out[:, rows].float()).all()
    assert float((s.out[:, rows].float() - want[:, rows].float()).abs().max()) <= 2.0 ** -6 * float(want.float().abs().max())
    assert bool(torch.isnan(s.out[:, n // 2].float()).all())


def test_tree_attn_in_place_is_refused(binding):
    s = Step(61, 4, 2, 64, 16, [(20, 3)])
    before = s.qd.clone()
    with pytest.raises(binding.SpError) as e:
        binding.Context().sp_tree_attn(s.qd, s.kd, s.vd, s.table_d, s.lens_d, s.start_d, s.qd)
    torch.cuda.synchronize()
    assert e.value.code == -1 and bool((s.qd == before).all())


@pytest.mark.parametrize("hq,hkv,d,page,reqs", [
    (8, 2, 128, 32, [(300, 1)] * 30 + [(500, 100)] + [(40, 2)] * 10),          # 400 rows among few: cut into units of 128
    (4, 4, 64, 16, [(900, 257), (300, 300)]), (4, 1, 128, 64, [(700, 65), (200, 64), (30, 1)]), (2, 1, 64, 16, [(5, 255), (900, 130)]),
])
def test_tree_attn_long_chunks_beside_single_tokens(attn_ctx, hq, hkv, d, page, reqs):
    s = Step(71, hq, hkv, d, page, reqs, "tree" if max(n for _, n in reqs) <= 256 else "chain", 2)
    s.call(attn_ctx)
    clean(attn_ctx)
    s.check()


@pytest.mark.parametrize("hq,d,new", [(4, 64, 10), (2, 128, 33)])
@pytest.mark.parametrize("rise", [40.0, -40.0], ids=["climbing", "falling"])
def test_tree_attn_levels_that_change_along_long_runs(attn_ctx, hq, d, new, rise):
    """Several tiles of 128 keys for every SM, each 40 nats above (below) the one before, eight in a row."""
    s = Step(19, hq, 2, d, 64, [(60000, new), (50, 2)], "tree", 1, "paged")
    s.q[..., 0] = 8.0
    x = np.arange(60000 + new)
    level = (x // 128 % 8) * rise
    s.k[s.table[0, x // 64], :, x % 64, 0] = torch.tensor(level * np.sqrt(d) / 8).to(torch.bfloat16).double().numpy()[:, None]
    s.qd, s.kd = dev(s.q).transpose(0, 1), dev(s.k)
    s.call(attn_ctx)
    clean(attn_ctx)
    out = host(s.out)
    off = d * 2.0 ** -23 * 7 * 40                                              # as above
    for h, rows, want, want_lse, tol in s.reference():
        assert np.all(np.abs(out[h, rows] - want) <= tol + 2 * off * np.abs(s.v).max())
    end = sum(n for _, n in s.reqs)
    assert np.all(out[:, end:] == 9)


def climb(s, step):
    """Gives key x of each request the level `step(x)` (in nats) through the first column; the farthest level."""
    s.q[..., 0] = 8.0
    far = 0.0
    for b, (p, n) in enumerate(s.reqs):
        for x in range(p + n):
            level = step(x)
            far = max(far, abs(level))
            s.k[s.table[b, x // s.page], :, x % s.page, 0] = float(torch.tensor(level * np.sqrt(s.d) / 8).to(torch.bfloat16))
    s.qd, s.kd = dev(s.q).transpose(0, 1), dev(s.k)
    return far


def close_to_reference(s, far):
    out = host(s.out)
    off = s.d * 2.0 ** -23 * far                                               # an fp32 sum of d terms of which one is `far` sqrt(d)
    for h, rows, want, want_lse, tol in s.reference():
        assert np.all(np.abs(out[h, rows] - want) <= tol + 2 * off * np.abs(s.v).max())


@pytest.mark.parametrize("hq,hkv,d,page,reqs", [(4, 1, 128, 16, [(700, 40), (3, 1)]), (2, 2, 64, 64, [(600, 130)]), (8, 2, 128, 128, [(1000, 64), (300, 50)]),
                                                (2, 2, 128, 32, [(500, 20)]), (2, 2, 64, 16, [(500, 3)])])
@pytest.mark.parametrize("rise", [9.0, 40.0])
def test_tree_attn_logits_that_climb_within_a_tile(attn_ctx, hq, hkv, d, page, reqs, rise):
    """Every 32 keys the maximum grows: references move in each chunk of a tile, with sums of earlier tiles and weights of
    the chunk before just written."""
    s = Step(23, hq, hkv, d, page, reqs, "tree", 1)
    far = climb(s, lambda x: x // 32 * rise)
    s.call(attn_ctx)
    clean(attn_ctx)
    close_to_reference(s, far)


@pytest.mark.parametrize("n_req,n", [(600, 1), (450, 40), (300, 200)], ids=["narrow", "tall", "wide"])
def test_tree_attn_long_waits_while_a_range_failure_has_not_been_read(binding, n_req, n):
    """A bad page of an earlier call stops nobody, not even waits of a millisecond (several requests of 128000 keys for each SM)."""
    ctx, fresh = binding.Context(), binding.Context()
    s = Step(31, 4, 2, 64, 16, [(100, 2), (50, 3)], "chain")
    s.table_d[0, 2] = -1
    s.call(ctx)
    g = torch.Generator(device="cuda").manual_seed(n)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)
    pages = 1002
    kc, vc, q = normal(pages, 1, 128, 64), normal(pages, 1, 128, 64), normal(1, n_req * n, 64)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(n_req, 1)           # all of them read the same pages
    lens, start = i32([128000 + n - b for b in range(n_req)]), i32([b * n for b in range(n_req + 1)])
    out, want = torch.zeros_like(q), torch.zeros_like(q)
    ctx.sp_tree_attn(q, kc, vc, table, lens, start, out)
    fresh.sp_tree_attn(q, kc, vc, table, lens, start, want)
    clean(fresh)
    assert ctx.status() == (binding.SP_ERR_RANGE, 70)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and bool((want != 0).any(-1).all())


def test_lengths_in_place_are_refused(binding):
    """Lengths that would be read and written by different blocks of one launch."""
    ctx = binding.Context()

    def refused(call, *args, **kw):
        before = [a.clone() if torch.is_tensor(a) else a for a in args]
        with pytest.raises(binding.SpError) as e:
            call(*args, **kw)
        torch.cuda.synchronize()
        assert e.value.code == -1 and all(torch.equal(a, b) for a, b in zip(args, before) if torch.is_tensor(a))

    def tables(**over):
        a = dict(past_lens=i32([3, 20]), new_lens=i32([2, 1]), page=16, free_pages=i32([5, 6, 7]), block_table=i32([[0, -1], [1, 2]]), seq_lens=i32([0, 0]),
                 row_start=i32([0] * 3), positions=i32([0] * 3), slots=i32([0] * 3), info=i32([0] * 4))
        a.update(over)
        return a
    lens, both, table = i32([3, 20]), i32([3, 20, 2, 1, 0]), i32([[0, -1], [1, 2]])
    for over in (dict(past_lens=lens, seq_lens=lens), dict(new_lens=lens, seq_lens=lens), dict(past_lens=both[:2], seq_lens=both[1:3]),
                 dict(new_lens=both[2:4], row_start=both[:3]), dict(positions=both[:3], slots=both[:3]), dict(free_pages=both, info=both[:4]),
                 dict(block_table=table, free_pages=table.view(-1)), dict(block_table=table, slots=table.view(-1)[:3])):
        refused(ctx.sp_page_tables, *tables(**over).values())
    parents = i32([-1, 0, -1])
    refused(ctx.sp_page_tables, *tables().values(), parents=parents, tree_mask=parents.view(3, 1))
    ctx.sp_page_tables(*tables(past_lens=both[:2], new_lens=both[2:4]).values())            # inputs may lie side by side
    kc, vc = (torch.zeros(3, 1, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kept = i32([[0, 1], [0, 1]])
    for past, n_kept, out in ((lens, i32([1, 1]), lens), (i32([3, 20]), lens, lens), (i32([3, 20]), i32([1, 1]), kept.view(-1)[2:]),
                              (i32([3, 20]), i32([1, 1]), table.view(-1)[:2])):
        refused(ctx.sp_cache_keep, kc, vc, table, past, kept, n_kept, out)
    clean(ctx)


def test_norm_rope_angles_at_any_position_and_frequency(binding):
    """Angles of millions of turns a position: the fraction of a turn has to come from all bits of the frequency."""
    from fractions import Fraction
    pi = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862089986280348253421170679, 10 ** 100)
    freq = [9.9e8, 1.2345678e6, 4321.1, 7.0, 1.0, 1e-3, 2.0 ** -40, 0.0]
    pos = [2 ** 31 - 1, 2 ** 31 - 2, 10 ** 9 + 7, 131071, 1, 0, -1, -(2 ** 31)]
    rng = np.random.default_rng(9)
    x = ref.bf16_values(rng, len(pos), 3, 64)
    q, k, v = (y.transpose(0, 1) for y in dev(x).split([1, 1, 1], 1))
    q_out, k_out, v_out = (torch.empty_like(y) for y in (q, k, v))
    ctx = binding.Context()
    ctx.sp_qk_norm_rope(q, k, v, i32(pos), torch.tensor(freq, dtype=torch.float64), q_out, k_out, v_out)
    clean(ctx)
    turns = np.array([[float(Fraction(f) * p / (2 * pi) % 1) for f in freq] for p in pos])       # exact, rounded once
    c, s = np.cos(2 * np.pi * turns), np.sin(2 * np.pi * turns)
    for got, y in ((q_out, x[:, 0]), (k_out, x[:, 1])):
        a, b = y[:, :8], y[:, 8:16]
        want, size = y.copy(), np.abs(y)
        want[:, :8], want[:, 8:16] = a * c - b * s, b * c + a * s
        size[:, :8] = size[:, 8:16] = np.abs(a) + np.abs(b)
        # as in the plain statement: the angle is off by under 2^-25 of a turn, its sine and cosine by under 2^-21
        assert np.all(np.abs(host(got)[0] - want) <= ref.EPS_BF16 * np.abs(want) + size * 2.0 ** -18)


def test_a_step_without_requests_is_no_work(binding):
    """Tensors without elements have no address."""
    ctx = binding.Context()
    none, ints = torch.empty(0, dtype=torch.int32, device="cuda"), lambda *shape: torch.full(shape, 5, dtype=torch.int32, device="cuda")
    start, info, pos, slots = ints(1), ints(4), ints(3), ints(3)
    ctx.sp_page_tables(none, none, 16, none, none.view(0, 4), none, start, pos, slots, info)
    ctx.sp_page_tables(none, none, 16, none, none.view(0, 4), none, start, none, none, info, parents=none, tree_mask=none.view(0, 1))
    kc, vc = (torch.ones(2, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for rows in (0, 3):
        q, out = (torch.ones(rows, 4, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2))
        ctx.sp_tree_attn(q, kc, vc, none.view(0, 4), none, start, out, lse_out=torch.ones(4, rows, device="cuda"))
        assert bool((out == 1).all())
    ctx.sp_cache_keep(kc, vc, none.view(0, 4), none, none.view(0, 3), none, none)
    clean(ctx)
    assert all(bool((x == 5).all()) for x in (start, info, pos, slots)) and bool((kc == 1).all()) and bool((vc == 1).all())


def test_cache_keep_of_nothing(binding):
    """No column of kept tokens: nothing moves, the lengths are those of before."""
    ctx = binding.Context()
    kc, vc = (torch.randn(3, 2, 16, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    before, lens = kc.clone(), i32([7, 7])
    ctx.sp_cache_keep(kc, vc, i32([[0], [1]]), i32([3, 0]), torch.empty(2, 0, dtype=torch.int32, device="cuda"), i32([0, 0]), lens)
    clean(ctx)
    assert lens.tolist() == [3, 0] and torch.equal(kc, before)


def test_tree_attn_mask_without_words_is_refused(binding):
    """Not taken for no mask at all, which means a chain."""
    s = Step(5, 4, 2, 64, 16, [(20, 3)])
    with pytest.raises(ValueError, match="tree_mask"):
        binding.Context().sp_tree_attn(s.qd, s.kd, s.vd, s.table_d, s.lens_d, s.start_d, s.out, tree_mask=torch.empty(s.rows, 0, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert bool((s.out == 9).all())


def test_wrong_shapes_are_named(binding):
    ctx, x, t = binding.Context(), i32([1, 2]), i32([[1, 2], [3, 4]])
    with pytest.raises(ValueError, match="^past_lens: expected one dimension$"):
        ctx.sp_page_tables(t, x, 16, x, t, x, i32([0] * 3), x, x, i32([0] * 4))
    with pytest.raises(ValueError, match="^new_lens: expected 2 elements in one dimension$"):
        ctx.sp_page_tables(x, i32([1, 2, 3]), 16, x, t, x, i32([0] * 3), x, x, i32([0] * 4))
    with pytest.raises(ValueError, match="^block_table: expected a two-dimensional tensor of 2 rows$"):
        ctx.sp_page_tables(x, x, 16, x, x, x, i32([0] * 3), x, x, i32([0] * 4))


# rows at which the streaming kernel of the rotation starts to hand whole tokens to its warps (148 x 16), several items a token
@pytest.mark.parametrize("hq,hkv,d,rows,n_freq,interleaved,norm,outs,page,major", [
    (8, 2, 128, 2367, 64, False, True, True, 16, True), (8, 2, 128, 2368, 64, False, True, True, 16, False), (8, 2, 128, 2369, 64, True, True, False, 64, True),
    (28, 4, 128, 5000, 64, False, True, True, 128, False), (24, 8, 64, 3001, 16, False, True, True, 32, True), (24, 8, 64, 4800, 32, True, False, True, 0, True)])
def test_norm_rope_of_many_rows(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, major):
    rope_case(binding, hq, hkv, d, rows, n_freq, interleaved, norm, outs, page, major, seed=rows)


@pytest.mark.parametrize("rows", [1000, 5000])
def test_norm_rope_of_many_rows_in_place(binding, rows):
    rng = np.random.default_rng(rows)
    x = ref.bf16_values(rng, rows, 12, 128)
    w = [ref.bf16_values(rng, 128) for _ in range(2)]
    freq = 5e5 ** (-np.arange(64) / 64.0)
    pos = rng.integers(0, 131072, rows)
    t = dev(x)
    q, k, v = (y.transpose(0, 1) for y in t.split([8, 2, 2], 1))
    ctx = binding.Context()
    ctx.sp_qk_norm_rope(q, k, v, i32(pos), torch.tensor(freq), q, k, v, q_weight=dev(w[0]), k_weight=dev(w[1]))
    clean(ctx)
    x = x.transpose(1, 0, 2)
    got = host(t).transpose(1, 0, 2)
    for heads, weight in ((slice(0, 8), w[0]), (slice(8, 10), w[1])):
        want, err = ref.norm_rope(x[heads], weight, 1e-6, freq, False, pos)
        assert np.all(np.abs(got[heads] - want) <= err + ref.EPS_BF16 * np.abs(want))
    assert np.array_equal(got[10:], x[10:])


def test_norm_rope_of_many_rows_with_slots_behind_the_cache(binding):
    rows, page, pages = 3000, 16, 100
    ctx = binding.Context()
    x = torch.randn(rows, 14, 128, device="cuda").to(torch.bfloat16)
    q, k, v = (y.transpose(0, 1) for y in x.split([8, 3, 3], 1))
    kc, vc = (torch.zeros(pages, 3, page, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = torch.full((rows,), -1, dtype=torch.int32)
    some = torch.randperm(rows)
    slots[some[:1000]] = torch.randperm(pages * page)[:1000].int()
    slots[some[1000:1100]] = pages * page + torch.arange(100, dtype=torch.int32) * 7
    ctx.sp_qk_norm_rope(q, k, v, i32(range(rows)), torch.zeros(0, dtype=torch.float64), torch.empty_like(q), k_cache=kc, v_cache=vc, slots=slots.cuda())
    torch.cuda.synchronize()
    assert ctx.status() == (binding.SP_ERR_RANGE, 75) and ctx.status() == (0, 0)
    for cache, y in ((kc, k), (vc, v)):
        want = torch.zeros(pages * page, 3, 128, dtype=torch.bfloat16, device="cuda")
        want[slots[some[:1000]].long().cuda()] = y.transpose(0, 1)[some[:1000].cuda()]
        assert torch.equal(cache.transpose(1, 2).reshape(-1, 3, 128), want)


@pytest.mark.parametrize("hq,hkv,d,page,reqs", [(8, 2, 128, 32, [(300, 9), (40, 1)]), (4, 4, 64, 256, [(700, 3), (90, 1)]), (4, 1, 128, 16, [(500, 70)])])
def test_tree_attn_of_other_orders(attn_ctx, hq, hkv, d, page, reqs):
    """Keys with the pages of a head side by side, values token-major, queries and results head-major and four-dimensional."""
    s = Step(81, hq, hkv, d, page, reqs, "tree", 2)
    total = s.k.shape[0]
    s.kd = dev(s.k.transpose(1, 0, 2, 3)).reshape(hkv, total * page, d).unflatten(1, (total, page)).transpose(0, 1)
    s.vd = dev(s.v.transpose(0, 2, 1, 3)).transpose(1, 2)
    s.qd = s.qd.contiguous().unsqueeze(0)
    s.out = torch.full((1, hq, s.rows, d), 9.0, dtype=torch.bfloat16, device="cuda")
    s.call(attn_ctx)
    clean(attn_ctx)
    s.out = s.out[0]
    s.check()


@pytest.mark.parametrize("d,page", [(64, 256), (128, 256), (128, 128)])
def test_tree_attn_far_references_with_pages_as_long_as_a_tile_or_longer(attn_ctx, d, page):
    """Runs that are walked again."""
    s = Step(83, 4, 2, d, page, [(2000, 10), (700, 20)], "tree", 1)
    far = climb(s, lambda x: x // 128 * 40.0)
    s.call(attn_ctx)
    clean(attn_ctx)
    close_to_reference(s, far)


def test_page_tables_with_an_empty_list_whose_address_is_anywhere(binding):
    """Through the C call: no free page and no row, their addresses inside another array of the call."""
    ctx = binding.Context()
    past, new, table, lens, start, info = i32([3, 20]), i32([0, 0]), i32([[0, -1], [1, 2]]), i32([0, 0]), i32([9] * 3), i32([9] * 4)
    inside = table.data_ptr() + 4
    code = binding.load().sp_page_tables(ctx._h, past.data_ptr(), new.data_ptr(), 2, 16, inside, 0, table.data_ptr(), 2, None, lens.data_ptr(), start.data_ptr(),
                                         inside, inside, None, 0, 0, info.data_ptr(), torch.cuda.current_stream().cuda_stream)
    clean(ctx)
    assert code == 0 and lens.tolist() == [3, 20] and start.tolist() == [0, 0, 0] and info.tolist() == [0, 0, 0, 20] and table.tolist() == [[0, -1], [1, 2]]
