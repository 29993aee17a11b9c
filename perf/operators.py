"""Cases and plain forms of the operators that carry a prompt from prefill into decoding.

Four operators, in the order in which a decoding step calls them:

  tables   request lengths (and, for a tree of drafted tokens, each token's parent) -> page tables that have grown to
           hold the new tokens, a cache slot and a position per token, the tree's visibility bits
  rope     norm of every query and key head, position rotation, and the move of q, k, v from the projection's
           token-major rows into head-major tensors and/or the paged cache
  attn     attention of a few new tokens per request (one, a chain or a tree) over the paged cache
  keep     after verification: the accepted tokens' keys and values move to the front of the drafted region

Layouts: q, k, v are [heads, tokens, head_dim] views with any strides, caches [pages, kv_heads, page, head_dim], all
bf16; tables, lengths, positions and slots are int32; the tokens of all requests are packed, request b owning rows
row_start[b] .. row_start[b + 1].  The lengths of a case are fixed by the case (dealt to its requests by the seed), so
that its work is too.

`run` is the plain form in elementary torch operations, 32 bits (64 for rotation angles), rounded once; with `own` set
it makes the library's calls.  `exact` states each operator again in 64 bits.
"""
import math
import random

import torch

own = False

EPS = 1e-6
THETA = 5e5
_context = None


def context():
    """The one library context that a serving process keeps."""
    global _context
    if _context is None:
        from paper_2505_19578_b200 import binding
        _context = binding.Context()
    return _context


# ---------------------------------------------------------------- cases

def listed():
    return [
        # a few chats, one token each: the smallest scheduling step, all latency
        dict(name="tables_chat", op="tables", requests=8, past_lo=40, past_hi=8000, new=1, tree=False, page=64, spare=8),
        # a full server that drafts trees: small pages, long tables, visibility bits of 64 drafted tokens
        dict(name="tables_trees", op="tables", requests=256, past_lo=100, past_hi=32768, new=64, tree=True, page=16, spare=0),
        # one token of one request in a layer of 32 query and 8 key heads, rotation only
        dict(name="rope_token", op="rope", hq=32, hkv=8, d=128, tokens=1, rot=128, norm=False, pairs="half", head_major=False, cache=True, page=64),
        # drafted trees of a batch: norms, rotation, keys and values into the cache
        dict(name="rope_trees", op="rope", hq=28, hkv=4, d=128, tokens=1000, rot=128, norm=True, pairs="half", head_major=False, cache=True, page=16),
        # a whole prompt: head-major q, k, v for the prefill call, and the cache
        dict(name="rope_prompt", op="rope", hq=32, hkv=8, d=128, tokens=131072, rot=128, norm=True, pairs="half", head_major=True, cache=True, page=128),
        # single tokens over a short cache, small heads: the least work a call can have
        dict(name="attn_short", op="attn", hq=8, hkv=8, d=64, requests=1, past_lo=2000, past_hi=2000, new=1, tree=False, page=64, pad=0),
        # one token after a full-length prompt: one request has to fill the device
        dict(name="attn_token_128k", op="attn", hq=32, hkv=8, d=128, requests=1, past_lo=131000, past_hi=131000, new=1, tree=False, page=128, pad=0),
        # a drafted tree of 64 after a full-length prompt: 256 rows per key head
        dict(name="attn_tree_128k", op="attn", hq=32, hkv=8, d=128, requests=1, past_lo=131000, past_hi=131000, new=64, tree=True, page=128, pad=0),
        # ragged batch with trees, seven query heads per key head, rows padded for a captured graph
        dict(name="attn_trees_ragged", op="attn", hq=28, hkv=4, d=128, requests=32, past_lo=700, past_hi=65536, new=16, tree=True, page=16, pad=9),
        # many short chats, one token each
        dict(name="attn_chats", op="attn", hq=32, hkv=8, d=128, requests=256, past_lo=60, past_hi=4000, new=1, tree=False, page=32, pad=0),
        # one accepted path
        dict(name="keep_one", op="keep", hkv=8, d=128, requests=1, past_lo=5000, past_hi=5000, new=16, kept=5, page=64),
        # a full server's accepted paths
        dict(name="keep_batch", op="keep", hkv=8, d=128, requests=256, past_lo=100, past_hi=4000, new=64, kept=12, page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "rope", "rope", "attn", "attn", "attn", "keep"])
    hq, hkv, d = rng.choice([(32, 8, 128), (28, 4, 128), (8, 8, 64), (8, 1, 128), (16, 4, 64)])
    page = rng.choice([16, 32, 64, 128])
    if op == "rope":
        pairs = rng.choice(["half", "half", "interleaved"])
        return dict(op=op, hq=hq, hkv=hkv, d=d, tokens=_log(rng, 1, 60000), rot=rng.choice([d, d, d // 2, 16]), norm=rng.random() < 0.6,
                    pairs=pairs, head_major=rng.random() < 0.5, cache=rng.random() < 0.8, page=page)
    requests = _log(rng, 1, 250)
    if op == "tables":
        lo = _log(rng, 1, 30000)
        return dict(op=op, requests=requests, past_lo=lo, past_hi=_log(rng, lo, 32000), new=_log(rng, 1, 64), tree=rng.random() < 0.6, page=page, spare=_log(rng, 1, 40))
    if op == "keep":
        lo = _log(rng, 1, 4000)
        new = _log(rng, 2, 64)
        return dict(op=op, hkv=hkv, d=d, requests=requests, past_lo=lo, past_hi=_log(rng, lo, 4000), new=new, kept=rng.randint(1, min(new, 16)), page=page)
    longest = min(131000, 240000 // requests)        # no more cached tokens, nor more pairs of token and key, than the largest listed case
    lo = _log(rng, 1, longest)
    hi = _log(rng, lo, longest)
    return dict(op=op, hq=hq, hkv=hkv, d=d, requests=requests, past_lo=lo, past_hi=hi, new=min(_log(rng, 1, 64), 8000000 // (requests * hi)), tree=rng.random() < 0.6,
                page=page, pad=rng.choice([0, 0, 7]))


def _lengths(case):
    """Cached and new tokens of each request, before the seed deals them out."""
    n, lo, hi = case["requests"], case["past_lo"], case["past_hi"]
    past = [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) for i in range(n)]
    new = [case["new"] - (5 * i) % max(1, case["new"] // 2) for i in range(n)]
    return past, new


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _dealt(case, seed):
    past, new = _lengths(case)
    order = list(range(len(past)))
    random.Random(seed).shuffle(order)
    return [past[i] for i in order], [new[i] for i in order]


def _paged(g, lens, page, width, n_pages):
    """A table of `width` pages per request whose first ceil(len / page) entries are taken from a random order of all
    pages, and the pages that are left, in that order."""
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    held = [-(-x // page) for x in lens]
    first = torch.tensor([sum(held[:i]) for i in range(len(held))], device="cuda")
    held = torch.tensor(held, device="cuda")
    col = torch.arange(width, device="cuda")
    at = first[:, None] + col
    table = torch.where(col < held[:, None], order[at.clamp(max=n_pages - 1)], torch.full_like(order[:1], -1))
    return table.contiguous(), order[int(held.sum()):].contiguous()


def _parents(case, new, seed):
    """Parent of each drafted token inside its request: the token before it or an earlier one (-1: the last cached token)."""
    r = random.Random(seed + 1)
    out = []
    for n in new:
        out += [max(-1, j - 1 - int(r.random() * r.random() * 8)) for j in range(n)]
    return out


def prepare(case, seed):
    g = _generator(seed)
    st = dict(case)
    if case["op"] == "rope":
        return _prepare_rope(st, case, g)
    page = case["page"]
    past, new = _dealt(case, seed)
    total = [p + n for p, n in zip(past, new)]
    width = -(-max(total) // page) + 2
    n_pages = sum(-(-t // page) for t in total) + 3
    st["past"], st["new_lens"] = _i32(past), _i32(new)
    if case["op"] == "tables":
        rows = sum(new) + case["spare"]
        st["table"], st["free"] = _paged(g, past, page, width, n_pages)
        st["parents"] = _i32(_parents(case, new, seed) + [-1] * case["spare"]) if case["tree"] else None
        st["seq_lens"], st["row_start"] = torch.zeros_like(st["past"]), _i32([0] * (len(past) + 1))
        st["positions"], st["slots"] = _i32([0] * rows), _i32([-1] * rows)
        st["bits"] = torch.zeros(rows, -(-case["new"] // 32), dtype=torch.int32, device="cuda") if case["tree"] else None
        st["info"] = _i32([0, 0, 0, 0])
        return st
    st["table"], _ = _paged(g, total, page, width, n_pages)
    shape = (n_pages, case["hkv"], page, case["d"])
    st["k_cache"], st["v_cache"] = _normal(g, *shape), _normal(g, *shape)
    if case["op"] == "keep":
        r = random.Random(seed + 2)
        counts = [min(r.randint(1, case["kept"]), n) for n in new]
        paths = [sorted(r.sample(range(n), c)) for n, c in zip(new, counts)]
        st["kept"] = _i32([p + [-1] * (case["kept"] - len(p)) for p in paths])
        st["n_kept"], st["lens_out"] = _i32(counts), torch.zeros_like(st["past"])
        return st
    rows = sum(new) + case["pad"]
    st["q"] = _normal(g, rows, case["hq"], case["d"]).mul_(1.5).transpose(0, 1)
    st["seq_lens"], st["row_start"] = _i32(total), _i32([sum(new[:i]) for i in range(len(new) + 1)])
    st["bits"] = None
    if case["tree"]:
        parents = _parents(case, new, seed)
        start = 0
        words = -(-case["new"] // 32)
        bits = []
        for n in new:
            seen = []
            for j in range(n):
                p = parents[start + j]
                seen.append((seen[p] if p >= 0 else 0) | 1 << j)
            bits += [[(s >> 32 * w) & 0xFFFFFFFF for w in range(words)] for s in seen]
            start += n
        bits += [[0] * words] * case["pad"]
        st["bits"] = torch.tensor(bits, dtype=torch.int64).cuda().to(torch.int32)
    st["out"] = torch.zeros(rows, case["hq"], case["d"], dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    st["lse"] = torch.zeros(case["hq"], rows, device="cuda")
    return st


def _prepare_rope(st, case, g):
    t, hq, hkv, d, page = case["tokens"], case["hq"], case["hkv"], case["d"], case["page"]
    qkv = _normal(g, t, hq + 2 * hkv, d)
    if case["norm"]:
        qkv.mul_(1 + 3 * torch.rand(hq + 2 * hkv, 1, generator=g, device="cuda").to(torch.bfloat16))
    st["q"], st["k"], st["v"] = (x.transpose(0, 1) for x in qkv.split([hq, hkv, hkv], dim=1))
    st["q_weight"], st["k_weight"] = ((1 + 0.3 * _normal(g, d), 1 + 0.3 * _normal(g, d)) if case["norm"] else (None, None))
    st["inv_freq"] = THETA ** (-torch.arange(case["rot"] // 2, dtype=torch.float64) * 2 / case["rot"])
    far = torch.randint(0, 131072, (t,), generator=g, device="cuda")
    st["positions"] = (torch.arange(t, device="cuda") if case["head_major"] else far).to(torch.int32)
    blank = torch.zeros if case["head_major"] else lambda h, n, e, **kw: torch.zeros(n, h, e, **kw).transpose(0, 1)
    kind = dict(dtype=torch.bfloat16, device="cuda")
    st["q_out"] = blank(hq, t, d, **kind)
    plain = case["head_major"] or not case["cache"]
    st["k_out"], st["v_out"] = (blank(hkv, t, d, **kind), blank(hkv, t, d, **kind)) if plain else (None, None)
    st["k_cache"] = st["v_cache"] = st["slots"] = None
    if case["cache"]:
        n_pages = -(-t // page) + 2
        st["k_cache"], st["v_cache"] = torch.zeros(n_pages, hkv, page, d, **kind), torch.zeros(n_pages, hkv, page, d, **kind)
        order = torch.randperm(n_pages, generator=g, device="cuda")
        at = torch.arange(t, device="cuda")
        st["slots"] = (order[at // page] * page + at % page).to(torch.int32)
    return st


# ---------------------------------------------------------------- plain forms

def _rows_of(row_start, rows):
    """Request and index inside it of each packed row, and whether the row is any request's."""
    t = torch.arange(rows, device="cuda")
    req = torch.searchsorted(row_start[1:].contiguous(), t, right=True).clamp(max=row_start.numel() - 2)
    return req, t - row_start[req], t < row_start[-1]


def _plain_tables(st):
    page, past, new, table, free = st["page"], st["past"].long(), st["new_lens"].long(), st["table"], st["free"]
    total = past + new
    held, need = (past + page - 1) // page, (total + page - 1) // page - (past + page - 1) // page
    first = need.cumsum(0) - need
    col = torch.arange(table.shape[1], device="cuda")
    at = first[:, None] + col - held[:, None]
    grown = (col >= held[:, None]) & (col < (held + need)[:, None])
    table.copy_(torch.where(grown, free[at.clamp(0, free.numel() - 1)], table))
    row_start = torch.cat([new.new_zeros(1), new.cumsum(0)])
    rows = st["slots"].numel()
    req, j, live = _rows_of(row_start, rows)
    p = past[req] + j
    slots = table[req, (p // page).clamp(max=table.shape[1] - 1)].long() * page + p % page
    depth = j
    if st["parents"] is not None:
        n = st["bits"].shape[1] * 32
        jc = torch.where(live, j, n)                                     # rows behind the last request go to a spare column
        par = torch.where(live, st["parents"].long(), -1)
        near = torch.zeros(len(past), n + 1, n + 1, device="cuda")
        near[req, jc, torch.where(par >= 0, par, jc)] = 1                # a token reaches its parent
        near[req, jc, jc] = 1                                            # and itself
        for _ in range(max(1, math.ceil(math.log2(n)))):                 # ... and, squared often enough, every ancestor
            near = (near @ near).clamp(max=1)
        seen = near[req, jc][:, :n]
        depth = seen.sum(1).long() - 1
        weight = 2 ** torch.arange(32, device="cuda")
        bits = (seen.view(rows, -1, 32).long() * weight).sum(2).to(torch.int32)
        st["bits"].copy_(torch.where(live[:, None], bits, st["bits"]))
    st["slots"].copy_(torch.where(live, slots.to(torch.int32), st["slots"]))
    st["positions"].copy_(torch.where(live, (past[req] + depth).to(torch.int32), st["positions"]))
    st["seq_lens"].copy_(total)
    st["row_start"].copy_(row_start)
    st["info"].copy_(torch.stack([row_start[-1], need.sum(), torch.zeros_like(need[0]), total.max()]))


def _turned(x, weight, cos, sin, st):
    """Norm and rotation of x [heads, tokens, d] in 32 bits."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    turn, rest = x[..., :st["rot"]], x[..., st["rot"]:]
    if st["pairs"] == "half":
        a, b = turn.chunk(2, -1)
        turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turn, rest], -1).to(torch.bfloat16)


def _plain_rope(st):
    angle = st["positions"].double()[:, None] * st["inv_freq"].cuda()
    cos, sin = angle.cos().float(), angle.sin().float()
    st["q_out"].copy_(_turned(st["q"], st["q_weight"], cos, sin, st))
    k = _turned(st["k"], st["k_weight"], cos, sin, st)
    if st["k_out"] is not None:
        st["k_out"].copy_(k)
        st["v_out"].copy_(st["v"])
    if st["k_cache"] is not None:
        page, off = st["slots"].long() // st["page"], st["slots"].long() % st["page"]
        st["k_cache"][page, :, off] = k.transpose(0, 1)
        st["v_cache"][page, :, off] = st["v"].transpose(0, 1)


def _plain_attn(st):
    hq, hkv, d, page = st["hq"], st["hkv"], st["d"], st["page"]
    rows, n_req, n = st["q"].shape[1], st["past"].numel(), st["new"]
    req, j, live = _rows_of(st["row_start"].long(), rows)
    pages = st["table"].clamp(min=0).long()
    keys = pages.shape[1] * page
    k = st["k_cache"][pages].float().permute(0, 2, 1, 3, 4).reshape(n_req, hkv, keys, d)
    # what lies behind a request's last token is not its own: zero, so that it adds nothing
    own_key = torch.arange(keys, device="cuda") < st["seq_lens"][:, None]
    v = st["v_cache"][pages].float().permute(0, 2, 1, 3, 4).reshape(n_req, hkv, keys, d)
    v = torch.where(own_key[:, None, :, None], v, 0)
    # rows of a request side by side: [request, token, heads], a spare token for the rows behind the last request
    q = torch.zeros(n_req, n + 1, hq, d, device="cuda")
    jc = torch.where(live, j, n)
    q[req, jc] = st["q"].transpose(0, 1).float()
    q = q.view(n_req, n + 1, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(n_req, hkv, -1, d)
    x = torch.arange(keys, device="cuda") - (st["seq_lens"] - st["row_start"].diff())[:, None]   # index among the new tokens
    seen = torch.zeros(n_req, n + 1, keys, dtype=torch.bool, device="cuda")
    if st["bits"] is None:
        seen[:] = x[:, None] <= torch.arange(n + 1, device="cuda")[:, None]
    else:
        bits = torch.zeros(n_req, n + 1, st["bits"].shape[1], dtype=torch.int64, device="cuda")
        bits[req, jc] = st["bits"].long()
        word = (x // 32).clamp(0, bits.shape[2] - 1)
        seen[:] = (bits.gather(2, word[:, None].expand(-1, n + 1, -1)) >> (x % 32)[:, None]) & 1 == 1
        seen |= x[:, None] < 0
    seen &= own_key[:, None]
    logits = (q @ k.transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(n_req, hkv, n + 1, -1, keys)
    logits.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = p.view(n_req, hkv, -1, keys) @ v / total.view(n_req, hkv, -1, 1).clamp(min=1e-30)
    out = out.view(n_req, hkv, n + 1, -1, d).permute(0, 2, 1, 3, 4).reshape(n_req, n + 1, hq, d)
    lse = (top + total.log()).permute(0, 2, 1, 3, 4).reshape(n_req, n + 1, hq)
    st["out"].copy_(torch.where(live[:, None], out[req, jc].transpose(0, 1).to(torch.bfloat16), st["out"]))
    st["lse"].copy_(torch.where(live, lse[req, jc].transpose(0, 1), st["lse"]))


def _plain_keep(st):
    page, kept = st["page"], st["kept"].long()
    i = torch.arange(kept.shape[1], device="cuda").expand_as(kept)
    live = i < st["n_kept"][:, None]
    req = torch.arange(len(kept), device="cuda")[:, None].expand_as(kept)[live]
    src, dst = ((st["past"].long()[:, None] + x)[live] for x in (kept, i))
    sp, dp = st["table"][req, src // page].long(), st["table"][req, dst // page].long()
    for cache in (st["k_cache"], st["v_cache"]):
        cache[dp, :, dst % page] = cache[sp, :, src % page]
    st["lens_out"].copy_(st["past"] + st["n_kept"])


# ---------------------------------------------------------------- one pass

def run(state):
    st = state
    op = st["op"]
    if op == "tables":
        if own:
            context().sp_page_tables(st["past"], st["new_lens"], st["page"], st["free"], st["table"], st["seq_lens"], st["row_start"],
                                     st["positions"], st["slots"], st["info"], parents=st["parents"], tree_mask=st["bits"])
        else:
            _plain_tables(st)
        return {k: st[k] for k in ("table", "seq_lens", "row_start", "positions", "slots", "bits", "info")}
    if op == "rope":
        if own:
            context().sp_qk_norm_rope(st["q"], st["k"], st["v"], st["positions"], st["inv_freq"], st["q_out"], k_out=st["k_out"], v_out=st["v_out"],
                                      k_cache=st["k_cache"], v_cache=st["v_cache"], slots=st["slots"], q_weight=st["q_weight"],
                                      k_weight=st["k_weight"], eps=EPS, interleaved=st["pairs"] == "interleaved")
        else:
            _plain_rope(st)
        return {k: st[k] for k in ("q_out", "k_out", "v_out", "k_cache", "v_cache")}
    if op == "attn":
        if own:
            context().sp_tree_attn(st["q"], st["k_cache"], st["v_cache"], st["table"], st["seq_lens"], st["row_start"], st["out"],
                                   tree_mask=st["bits"], lse_out=st["lse"])
        else:
            _plain_attn(st)
        return {"out": st["out"], "lse": st["lse"]}
    if own:
        context().sp_cache_keep(st["k_cache"], st["v_cache"], st["table"], st["past"], st["kept"], st["n_kept"], st["lens_out"])
    else:
        _plain_keep(st)
    return {"k_cache": st["k_cache"], "v_cache": st["v_cache"], "lens": st["lens_out"]}


def work(case):
    op = case["op"]
    if op == "rope":
        heads, t, d = case["hq"] + 2 * case["hkv"], case["tokens"], case["d"]
        stores = case["hq"] + 2 * case["hkv"] * ((case["head_major"] or not case["cache"]) + case["cache"])
        turned = t * (case["hq"] + case["hkv"]) * d
        return {"bytes": 2 * t * d * (heads + stores) + 4 * t * (1 + case["cache"]), "flops": turned * (3 + 4 * case["norm"])}
    past, new = _lengths(case)
    n = case["requests"]
    if op == "tables":
        page, rows = case["page"], sum(new)
        grown = sum(-(-(p + m) // page) - -(-p // page) for p, m in zip(past, new))
        per_row = 8 + case["tree"] * (4 + 4 * -(-case["new"] // 32))
        return {"bytes": 4 * (4 * n + 2 * grown + 4) + rows * per_row, "flops": 4 * rows}
    if op == "keep":
        # about half of the longest path is accepted; each token's K and V of every head is read and written
        moved = n * (case["kept"] + 1) / 2
        return {"bytes": moved * case["hkv"] * case["d"] * 2 * 2 * 2, "flops": moved}
    rows, keys = sum(new), sum(p + m for p, m in zip(past, new))
    pairs = sum((p + m) * m for p, m in zip(past, new)) * case["hq"]
    return {"bytes": keys * case["hkv"] * case["d"] * 4 + rows * case["hq"] * (case["d"] * 4 + 4) + 4 * keys / case["page"], "flops": pairs * case["d"] * 4}


# ---------------------------------------------------------------- 64 bits

def _exact_attn(case, st):
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    out, lse = st["out"].double().clone(), st["lse"].double().clone()
    starts, lens = st["row_start"].tolist(), st["seq_lens"].tolist()
    table, bits = st["table"].tolist(), None if st["bits"] is None else st["bits"].tolist()
    for b, (s, e, length) in enumerate(zip(starts, starts[1:], lens)):
        ids = torch.tensor(table[b][:-(-length // page)], device="cuda")
        keys, values = (c[ids].transpose(0, 1).reshape(hkv, -1, d)[:, :length].double() for c in (st["k_cache"], st["v_cache"]))
        seen = torch.ones(e - s, length, dtype=torch.bool)
        for j in range(e - s):
            row = [x <= j if bits is None else bool(bits[s + j][x // 32] >> x % 32 & 1) for x in range(e - s)]
            seen[j, length - (e - s):] = torch.tensor(row)
        seen = seen.cuda()
        for h in range(hq):
            z = st["q"][h, s:e].double() @ keys[h * hkv // hq].T / d ** 0.5
            z[~seen] = -math.inf
            lse[h, s:e] = z.logsumexp(-1)
            out[h, s:e] = z.softmax(-1) @ values[h * hkv // hq]
    return {"out": out, "lse": lse}


def _exact_rope(case, st):
    rot, half = case["rot"], case["pairs"] == "half"
    phase = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["positions"].double()[:, None] * st["inv_freq"].cuda())

    def turned(x, weight):
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for h in range(x.shape[0]):
            z = x[h].double()
            if weight is not None:
                z = z * weight.double() / (z.pow(2).sum(-1, keepdim=True) / case["d"] + EPS).sqrt()
            even, odd = (slice(0, rot // 2), slice(rot // 2, rot)) if half else (slice(0, rot, 2), slice(1, rot, 2))
            c = torch.complex(z[:, even], z[:, odd]) * phase
            z[:, even], z[:, odd] = c.real, c.imag
            y[h] = z
        return y

    q, k, v = turned(st["q"], st["q_weight"]), turned(st["k"], st["k_weight"]), st["v"].double()
    got = {"q_out": q, "k_out": None, "v_out": None, "k_cache": None, "v_cache": None}
    if st["k_out"] is not None:
        got["k_out"], got["v_out"] = k, v
    if case["cache"]:
        slot = st["slots"].long()
        for name, x in (("k_cache", k), ("v_cache", v)):
            flat = st[name].double().transpose(1, 2).flatten(0, 1)            # [slot, head, d]
            flat[slot] = x.transpose(0, 1)
            got[name] = flat.unflatten(0, (-1, case["page"])).transpose(1, 2).contiguous()
    return got


def _exact_keep(case, st):
    past, kept, count, table = (st[k].tolist() for k in ("past", "kept", "n_kept", "table"))
    moves = []
    for b, n in enumerate(count):
        at = [(table[b][p // case["page"]], p % case["page"]) for p in range(past[b], past[b] + case["new"])
              if p // case["page"] < len(table[b])]
        moves += [(at[kept[b][i]], at[i]) for i in range(n)]
    got = {"lens": None}
    for name in ("k_cache", "v_cache"):
        new = st[name].double()
        for (sp, so), (dp, do) in moves:
            new[dp, :, do] = st[name][sp, :, so].double()
        got[name] = new
    return got


def exact(case, seed):
    if case["op"] == "tables":
        return None                                   # whole numbers only
    st = prepare(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "keep": _exact_keep}[case["op"]](case, st)
