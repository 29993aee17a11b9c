"""Cases and plain forms of the operators of a paged cache held in 4 bits.

Four operators, in the order in which a serving process calls them:

  append   norm of every query and key head, position rotation, and keys and values as 4-bit codes with a scale for each 32
           into the paged cache; then what was stored is read back (the next chunk's prefill reads it so)
  attn     attention of a few new tokens per request (one, a chain or a tree) over the cache
  keep     after verification: the accepted tokens' codes and scales move to the front of the drafted region, which is read back
  read     a cached prefix as head-major keys and values, as the prefill call takes them

A cache is uint8 [pages, kv_heads, page * 17 * head_dim / 16]: runs of blocks of 16 tokens.  A code c stands for (c - 8) * s,
a scale byte for s = (1 + low 3 bits / 8) * 2^(high 5 bits - 20).  Where a token's bytes lie in its block: `_layout`.

q, k, v are [heads, tokens, head_dim] views with any strides in bf16; tables, lengths, positions and slots are int32; the
tokens of all requests are packed, request b owning rows row_start[b] .. row_start[b + 1].  The lengths of a case are fixed
by the case (dealt to its requests by the seed), so that its work is too.

`run` is the plain form in elementary torch operations, 32 bits (64 for rotation angles, and for the keys on their way to
codes: next to a border between two codes 32 bits choose the wrong one), rounded once; with `own` set it makes the
library's calls.  `exact` states each operator again in 64 bits.
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
        # one token of one request in a layer of 32 query and 8 key heads, rotation only: all latency
        dict(name="append_token", op="append", hq=32, hkv=8, d=128, tokens=1, rot=128, norm=False, pairs="half", head_major=False, page=64),
        # drafted trees of a batch: norms, rotation, small pages
        dict(name="append_trees", op="append", hq=28, hkv=4, d=128, tokens=1000, rot=128, norm=True, pairs="half", head_major=False, page=16),
        # a whole prompt, queries head-major for the prefill call
        dict(name="append_prompt", op="append", hq=32, hkv=8, d=128, tokens=131072, rot=128, norm=True, pairs="half", head_major=True, page=128),
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
        # a chat's history before its next turn
        dict(name="read_turn", op="read", hkv=8, d=128, requests=1, past_lo=5001, past_hi=5001, page=64),
        # the prefixes of a batch of long documents
        dict(name="read_documents", op="read", hkv=4, d=128, requests=8, past_lo=3000, past_hi=131000, page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attn", "attn", "attn", "attn", "keep", "read"])
    hq, hkv, d = rng.choice([(32, 8, 128), (28, 4, 128), (8, 8, 64), (8, 1, 128), (16, 4, 64)])
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        pairs = rng.choice(["half", "half", "interleaved"])
        return dict(op=op, hq=hq, hkv=hkv, d=d, tokens=_log(rng, 1, 60000), rot=rng.choice([d, d, d // 2, 16]), norm=rng.random() < 0.6,
                    pairs=pairs, head_major=rng.random() < 0.5, page=page)
    requests = _log(rng, 1, 250)
    if op == "keep":
        lo = _log(rng, 1, 4000)
        new = _log(rng, 2, 64)
        return dict(op=op, hkv=hkv, d=d, requests=requests, past_lo=lo, past_hi=_log(rng, lo, 4000), new=new, kept=rng.randint(1, min(new, 16)), page=page)
    longest = min(131000, 240000 // requests)        # no more cached tokens, nor more pairs of token and key, than the largest listed case
    lo = _log(rng, 1, longest)
    hi = _log(rng, lo, longest)
    if op == "read":
        return dict(op=op, hkv=hkv, d=d, requests=requests, past_lo=lo, past_hi=hi, page=page)
    return dict(op=op, hq=hq, hkv=hkv, d=d, requests=requests, past_lo=lo, past_hi=hi, new=min(_log(rng, 1, 64), 8000000 // (requests * hi)), tree=rng.random() < 0.6,
                page=page, pad=rng.choice([0, 0, 7]))


def _lengths(case):
    """Cached and new tokens of each request, before the seed deals them out."""
    n, lo, hi, m = case["requests"], case["past_lo"], case["past_hi"], case.get("new", 0)
    past = [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) for i in range(n)]
    new = [m - (5 * i) % max(1, m // 2) for i in range(n)]
    return past, new


# ---------------------------------------------------------------- the format

_layouts = {}


def _layout(d):
    """[16, d + d / 16]: where, in a block of 16 tokens, token i has its K code bytes, V code bytes, K scales and V scales.
    Codes: a token's K bytes together, V by 64 elements and in an order of tokens; scales: K by token modulo 8, group, token / 8;
    V by group, then four bytes for tokens 2 j, 2 j + 8, 2 j + 1, 2 j + 9."""
    if d not in _layouts:
        i, b, g = torch.arange(16)[:, None], torch.arange(d // 2)[None], torch.arange(d // 32)[None]
        k = i * (d // 2) + b
        v = 8 * d + b // 32 * 512 + ((i & 8) | (i & 1) << 2 | (i & 7) >> 1) * 32 + b % 32
        ks = 16 * d + i % 8 * (d // 16) + 2 * g + i // 8
        vs = 16 * d + d // 2 + 16 * g + (i % 8 // 2 * 4 + i // 8 + i % 2 * 2)
        _layouts[d] = torch.cat([k, v, ks, vs], 1).cuda()
    return _layouts[d]


_ORDER = (0, 2, 4, 6, 1, 3, 5, 7)      # elements of a 32-bit word, from its lowest four bits up


def _page_bytes(page, d):
    return page * 17 * d // 16


def _coded(x):
    """x [..., d] -> codes as bytes [..., d / 2] and scale bytes [..., d / 32]; computed in x's type."""
    g = x.unflatten(-1, (-1, 32))
    a = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a / torch.full_like(a, 7))                    # (a division by a number would be a product with 1 / 7)
    s = torch.ldexp(torch.round(m * 16) / 16, e).clamp(2.0 ** -20, 1.875 * 2 ** 11)
    c = (torch.round(g / s).clamp(-7, 7) + 8).to(torch.uint8)
    m, e = torch.frexp(s.squeeze(-1))
    scale = ((e + 19) * 8 + (m * 16 - 8).to(e.dtype)).to(torch.uint8)
    n = c.flatten(-2).unflatten(-1, (-1, 8))[..., _ORDER].unflatten(-1, (4, 2))
    return (n[..., 0] + n[..., 1] * 16).flatten(-2), scale


def _decoded(codes, scale):
    """The values, in 32 bits (which hold them exactly)."""
    n = torch.stack([codes & 15, codes >> 4], -1).unflatten(-2, (-1, 4)).flatten(-2)        # [..., words, 8]
    n = n[..., (0, 4, 1, 5, 2, 6, 3, 7)].flatten(-2).float() - 8
    s = torch.ldexp(1 + (scale & 7).float() / 8, (scale >> 3).int() - 20)
    return (n.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _kv_of(rows, d):
    """Bytes of tokens [..., d + d / 16] -> keys and values [..., d]."""
    k, v, ks, vs = rows.split([d // 2, d // 2, d // 32, d // 32], -1)
    return _decoded(k, ks), _decoded(v, vs)


def _places(cache, page_ids, in_page, page, d):
    """[..., heads, d + d / 16]: indices of tokens' bytes in the flat cache."""
    head = torch.arange(cache.shape[1], device="cuda")
    at = (page_ids.long()[..., None] * cache.shape[1] + head) * cache.shape[2] + (in_page // 16 * (17 * d))[..., None]
    return at[..., None] + _layout(d)[in_page % 16][..., None, :]


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
    """A table of `width` pages per request whose first ceil(len / page) entries are taken from a random order of all pages."""
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    held = [-(-x // page) for x in lens]
    first = torch.tensor([sum(held[:i]) for i in range(len(held))], device="cuda")
    held = torch.tensor(held, device="cuda")
    col = torch.arange(width, device="cuda")
    at = first[:, None] + col
    return torch.where(col < held[:, None], order[at.clamp(max=n_pages - 1)], torch.full_like(order[:1], -1)).contiguous()


def _filled(g, n_pages, hkv, page, d):
    """A cache of coded keys (with channels that are larger than others, as keys have them) and values."""
    cache = torch.empty(n_pages * hkv, page // 16, 17 * d, dtype=torch.uint8, device="cuda")
    channel = torch.where(torch.rand(hkv, d, generator=g, device="cuda") < 0.05, 4.0, 1.0).to(torch.bfloat16)
    for lo in range(0, n_pages, 4096):                               # a slice at a time, for the temporaries' sake
        hi = min(lo + 4096, n_pages)
        k = _normal(g, hi - lo, hkv, page // 16, 16, d) * channel[None, :, None, None]
        v = _normal(g, hi - lo, hkv, page // 16, 16, d)
        (kc, ks), (vc, vs) = _coded(k.float()), _coded(v.float())
        rows = torch.cat([kc, vc, ks, vs], -1).flatten(0, 1).flatten(-2)
        part = torch.empty(rows.shape, dtype=torch.uint8, device="cuda")
        part[..., _layout(d).flatten()] = rows
        cache[lo * hkv:hi * hkv] = part
    return cache.view(n_pages, hkv, _page_bytes(page, d))


def _parents(case, new, seed):
    """Parent of each drafted token inside its request: the token before it or an earlier one (-1: the last cached token)."""
    r = random.Random(seed + 1)
    out = []
    for n in new:
        out += [max(-1, j - 1 - int(r.random() * r.random() * 8)) for j in range(n)]
    return out


def _starts(lens):
    return _i32([sum(lens[:i]) for i in range(len(lens) + 1)])


def _blank(heads, rows, d, head_major=True):
    kind = dict(dtype=torch.bfloat16, device="cuda")
    return torch.zeros(heads, rows, d, **kind) if head_major else torch.zeros(rows, heads, d, **kind).transpose(0, 1)


def prepare(case, seed):
    g = _generator(seed)
    st = dict(case)
    if case["op"] == "append":
        return _prepare_append(st, case, g)
    page, hkv, d = case["page"], case["hkv"], case["d"]
    past, new = _dealt(case, seed)
    total = [p + n for p, n in zip(past, new)]
    width = -(-max(total) // page) + 2
    n_pages = sum(-(-t // page) for t in total) + 3
    st["past"], st["seq_lens"] = _i32(past), _i32(total)
    st["table"] = _paged(g, total, page, width, n_pages)
    st["cache"] = _filled(g, n_pages, hkv, page, d)
    if case["op"] == "read":
        st["row_start"] = _starts(total)
        st["k"], st["v"] = _blank(hkv, sum(total), d), _blank(hkv, sum(total), d)
        return st
    st["row_start"] = _starts(new)
    if case["op"] == "keep":
        r = random.Random(seed + 2)
        counts = [min(r.randint(1, case["kept"]), n) for n in new]
        paths = [sorted(r.sample(range(n), c)) for n, c in zip(new, counts)]
        st["kept"] = _i32([p + [-1] * (case["kept"] - len(p)) for p in paths])
        st["n_kept"], st["lens_out"] = _i32(counts), torch.zeros_like(st["past"])
        st["k"], st["v"] = _blank(hkv, sum(new), d), _blank(hkv, sum(new), d)
        return st
    rows = sum(new) + case["pad"]
    st["q"] = _normal(g, rows, case["hq"], d).mul_(1.5).transpose(0, 1)
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
    st["out"] = _blank(case["hq"], rows, d, False)
    st["lse"] = torch.zeros(case["hq"], rows, device="cuda")
    return st


def _prepare_append(st, case, g):
    t, hq, hkv, d, page = case["tokens"], case["hq"], case["hkv"], case["d"], case["page"]
    qkv = _normal(g, t, hq + 2 * hkv, d)
    if case["norm"]:
        qkv.mul_(1 + 3 * torch.rand(hq + 2 * hkv, 1, generator=g, device="cuda").to(torch.bfloat16))
    st["q_in"], st["k_in"], st["v_in"] = (x.transpose(0, 1) for x in qkv.split([hq, hkv, hkv], dim=1))
    st["q_weight"], st["k_weight"] = ((1 + 0.3 * _normal(g, d), 1 + 0.3 * _normal(g, d)) if case["norm"] else (None, None))
    st["inv_freq"] = THETA ** (-torch.arange(case["rot"] // 2, dtype=torch.float64) * 2 / case["rot"])
    far = torch.randint(0, 131072, (t,), generator=g, device="cuda")
    st["positions"] = (torch.arange(t, device="cuda") if case["head_major"] else far).to(torch.int32)
    st["q_out"] = _blank(hq, t, d, case["head_major"])
    n_pages = -(-t // page) + 2
    st["table"] = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)[None].contiguous()
    at = torch.arange(t, device="cuda")
    st["slots"] = (st["table"][0, at // page] * page + at % page).to(torch.int32)
    st["cache"] = torch.zeros(n_pages, hkv, _page_bytes(page, d), dtype=torch.uint8, device="cuda")
    st["seq_lens"], st["row_start"] = _i32([t]), _i32([0, t])
    st["k"], st["v"] = _blank(hkv, t, d), _blank(hkv, t, d)
    return st


# ---------------------------------------------------------------- plain forms

def _rows_of(row_start, rows):
    """Request and index inside it of each packed row, and whether the row is any request's."""
    t = torch.arange(rows, device="cuda")
    req = torch.searchsorted(row_start[1:].contiguous(), t, right=True).clamp(max=row_start.numel() - 2)
    return req, t - row_start[req], t < row_start[-1]


def _turned(x, weight, cos, sin, st):
    """Norm and rotation of x [heads, tokens, d], in cos's type."""
    x = x.to(cos.dtype)
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.to(cos.dtype)
    turn, rest = x[..., :st["rot"]], x[..., st["rot"]:]
    if st["pairs"] == "half":
        a, b = turn.chunk(2, -1)
        turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turn, rest], -1)


def _plain_append(st):
    page, d = st["page"], st["d"]
    angle = st["positions"].double()[:, None] * st["inv_freq"].cuda()
    cos, sin = angle.cos(), angle.sin()
    st["q_out"].copy_(_turned(st["q_in"], st["q_weight"], cos.float(), sin.float(), st))
    kc, ks = _coded(_turned(st["k_in"], st["k_weight"], cos, sin, st).transpose(0, 1))
    vc, vs = _coded(st["v_in"].transpose(0, 1).float())
    slots = st["slots"].long()
    st["cache"].view(-1)[_places(st["cache"], slots // page, slots % page, page, d)] = torch.cat([kc, vc, ks, vs], -1)
    _plain_read(st)


def _plain_read(st):
    page, d = st["page"], st["d"]
    req, j, live = _rows_of(st["row_start"].long(), st["k"].shape[1])
    p = st["seq_lens"].long()[req] - st["row_start"].long().diff()[req] + j
    bytes_ = st["cache"].view(-1)[_places(st["cache"], st["table"][req, p // page], p % page, page, d)]       # [rows, heads, ...]
    k, v = _kv_of(bytes_, d)
    st["k"].copy_(k.transpose(0, 1))
    st["v"].copy_(v.transpose(0, 1))


def _plain_attn(st):
    hq, hkv, d, page = st["hq"], st["hkv"], st["d"], st["page"]
    rows, n_req, n = st["q"].shape[1], st["past"].numel(), st["new"]
    req, j, live = _rows_of(st["row_start"].long(), rows)
    pages = st["table"].clamp(min=0).long()
    keys = pages.shape[1] * page
    blocks = st["cache"][pages].transpose(1, 2).unflatten(-1, (page // 16, -1))                        # [n, heads, pages, blocks, bytes]
    bytes_ = blocks[..., _layout(d).flatten()].unflatten(-1, (16, -1)).flatten(2, 4)                     # [n, heads, keys, ...]
    del blocks
    k, v = _kv_of(bytes_, d)
    del bytes_
    own_key = torch.arange(keys, device="cuda") < st["seq_lens"][:, None]
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
    page, d, kept = st["page"], st["d"], st["kept"].long()
    i = torch.arange(kept.shape[1], device="cuda").expand_as(kept)
    live = i < st["n_kept"][:, None]
    req = torch.arange(len(kept), device="cuda")[:, None].expand_as(kept)[live]
    src, dst = ((st["past"].long()[:, None] + x)[live] for x in (kept, i))
    src, dst = (_places(st["cache"], st["table"][req, p // page], p % page, page, d) for p in (src, dst))
    flat = st["cache"].view(-1)
    flat[dst] = flat[src]
    st["lens_out"].copy_(st["past"] + st["n_kept"])
    _plain_read(st)


# ---------------------------------------------------------------- one pass

def run(state):
    st = state
    op = st["op"]
    if op == "append":
        if own:
            context().sp_qk_norm_rope_q4(st["q_in"], st["k_in"], st["v_in"], st["positions"], st["inv_freq"], st["q_out"], st["cache"], st["slots"],
                                         q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, interleaved=st["pairs"] == "interleaved")
            context().sp_cache_read_q4(st["cache"], st["table"], st["seq_lens"], st["row_start"], st["k"], st["v"])
        else:
            _plain_append(st)
        return {k: st[k] for k in ("q_out", "k", "v")}
    if op == "attn":
        if own:
            context().sp_tree_attn_q4(st["q"], st["cache"], st["table"], st["seq_lens"], st["row_start"], st["out"], tree_mask=st["bits"], lse_out=st["lse"])
        else:
            _plain_attn(st)
        return {"out": st["out"], "lse": st["lse"]}
    if op == "keep":
        if own:
            context().sp_cache_keep_q4(st["cache"], st["table"], st["past"], st["kept"], st["n_kept"], st["lens_out"], st["d"])
            context().sp_cache_read_q4(st["cache"], st["table"], st["seq_lens"], st["row_start"], st["k"], st["v"])
        else:
            _plain_keep(st)
        return {"k": st["k"], "v": st["v"], "lens": st["lens_out"]}
    if own:
        context().sp_cache_read_q4(st["cache"], st["table"], st["seq_lens"], st["row_start"], st["k"], st["v"])
    else:
        _plain_read(st)
    return {"k": st["k"], "v": st["v"]}


def work(case):
    op, d, hkv = case["op"], case["d"], case["hkv"]
    coded = 2 * hkv * (d // 2 + d // 32)                             # bytes of a token in the cache,
    full = 4 * hkv * d                                               # and as bf16 keys and values
    if op == "append":
        hq, t = case["hq"], case["tokens"]
        turned = t * (hq + hkv) * d
        return {"bytes": t * (4 * hq * d + full + coded + 8) + t * (coded + full), "flops": turned * (3 + 4 * case["norm"]) + 4 * t * hkv * d}
    past, new = _lengths(case)
    if op == "read":
        return {"bytes": sum(past) * (coded + full + 4 / case["page"]), "flops": 2 * sum(past) * hkv * d}
    if op == "keep":
        # about half of the longest path is accepted; each token's bytes of every head are read and written
        moved = case["requests"] * (case["kept"] + 1) / 2
        return {"bytes": 2 * moved * coded + sum(new) * (coded + full), "flops": 2 * sum(new) * hkv * d}
    rows, keys = sum(new), sum(p + m for p, m in zip(past, new))
    pairs = sum((p + m) * m for p, m in zip(past, new)) * case["hq"]
    return {"bytes": keys * coded + rows * case["hq"] * (d * 4 + 4) + 4 * keys / case["page"], "flops": pairs * d * 4}


# ---------------------------------------------------------------- 64 bits

def _exact_token_bytes(cache, ids, offs, d):
    """Of tokens (page ids and places in the page, host lists or device tensors): codes [tokens, heads, 2, d] and scale bytes
    [tokens, heads, 2, d / 32], picked out of the blocks field by field."""
    ids, offs = (torch.as_tensor(x, device="cuda").long() for x in (ids, offs))
    block = cache.unflatten(-1, (-1, 17 * d))[ids, :, offs // 16]                        # [tokens, heads, bytes]
    i = offs % 16
    t = torch.arange(len(ids), device="cuda")
    k = block[..., :8 * d].unflatten(-1, (16, d // 2))[t, :, i]
    v = block[..., 8 * d:16 * d].unflatten(-1, (d // 64, 16, 32))[t, :, :, (i // 8) * 8 + (i % 2) * 4 + i % 8 // 2].flatten(-2)
    ks = block[..., 16 * d:16 * d + d // 2].unflatten(-1, (8, d // 32, 2))[t, :, i % 8, :, i // 8]
    vs = block[..., 16 * d + d // 2:].unflatten(-1, (d // 32, 4, 2, 2))[t, :, :, i % 8 // 2, i % 2, i // 8]
    word = torch.stack([k, v], 2).contiguous().view(torch.int32).long()
    codes = torch.stack([word >> (4 * (e // 2) + 16 * (e % 2)) & 15 for e in range(8)], -1).flatten(-2)
    return codes, torch.stack([ks, vs], 2)


def _exact_values(codes, scales):
    s = (8 + scales % 8).double() * torch.pow(2.0, scales.double().div(8).floor() - 23)
    return (codes.double() - 8) * s.repeat_interleave(32, -1)


def _exact_rows(st, b, lo, hi):
    """Keys and values [heads, tokens, d] of tokens lo .. hi - 1 of request b."""
    p = torch.arange(lo, hi, device="cuda")
    kv = _exact_values(*_exact_token_bytes(st["cache"], st["table"][b][p // st["page"]], p % st["page"], st["d"]))
    return kv[:, :, 0].transpose(0, 1), kv[:, :, 1].transpose(0, 1)


def _exact_attn(case, st):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out, lse = st["out"].double().clone(), st["lse"].double().clone()
    starts, lens = st["row_start"].tolist(), st["seq_lens"].tolist()
    bits = None if st["bits"] is None else st["bits"].tolist()
    for b, (s, e, length) in enumerate(zip(starts, starts[1:], lens)):
        keys, values = _exact_rows(st, b, 0, length)
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


def _exact_rounded(x):
    """What codes and scales make of x [tokens, d], in 64 bits: the candidates of the scale are compared, not rounded."""
    g = x.unflatten(-1, (-1, 32))
    a = g.abs().amax(-1)
    a = a / torch.full_like(a, 7)
    e = a.clamp(2.0 ** -20, 1.875 * 2 ** 11).log2().floor()
    e = torch.where(torch.pow(2.0, e + 1) <= a, e + 1, torch.where(torch.pow(2.0, e) > a, e - 1, e)).clamp(-20, 11)
    s = torch.full_like(a, math.inf)
    for m in range(8, 17):                                           # 16: the next power of two
        c = m / 8 * torch.pow(2.0, e)
        c = torch.where(c > 1.875 * 2 ** 11, 1.875 * 2 ** 11, c)
        near, was = (c - a).abs(), (s - a).abs()
        s = torch.where((near < was) | ((near == was) & (m % 2 == 0)), c, s)
    return ((g / s[..., None]).round().clamp(-7, 7) * s[..., None]).flatten(-2)


def _exact_append(case, st):
    rot, half = case["rot"], case["pairs"] == "half"
    phase = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["positions"].double()[:, None] * st["inv_freq"].cuda())

    def turned(x, weight, rounded):
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for h in range(x.shape[0]):
            z = x[h].double()
            if weight is not None:
                z = z * weight.double() / (z.pow(2).sum(-1, keepdim=True) / case["d"] + EPS).sqrt()
            even, odd = (slice(0, rot // 2), slice(rot // 2, rot)) if half else (slice(0, rot, 2), slice(1, rot, 2))
            c = torch.complex(z[:, even], z[:, odd]) * phase
            z[:, even], z[:, odd] = c.real, c.imag
            y[h] = _exact_rounded(z) if rounded else z
        return y

    v = torch.stack([_exact_rounded(x.double()) for x in st["v_in"]])
    return {"q_out": turned(st["q_in"], st["q_weight"], False), "k": turned(st["k_in"], st["k_weight"], True), "v": v}


def _exact_read(case, st):
    starts, lens = st["row_start"].tolist(), st["seq_lens"].tolist()
    kv = [_exact_rows(st, b, n - (e - s), n) for b, (s, e, n) in enumerate(zip(starts, starts[1:], lens))]
    return {"k": torch.cat([k for k, _ in kv], 1), "v": torch.cat([v for _, v in kv], 1)}


def _exact_keep(case, st):
    got = _exact_read(case, st)
    starts, kept, count = st["row_start"].tolist(), st["kept"].tolist(), st["n_kept"].tolist()
    for x in got.values():
        old = x.clone()
        for b, n in enumerate(count):
            x[:, starts[b]:starts[b] + n] = old[:, [starts[b] + j for j in kept[b][:n]]]
    return {**got, "lens": None}


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "read": _exact_read, "keep": _exact_keep}[case["op"]](case, st)
