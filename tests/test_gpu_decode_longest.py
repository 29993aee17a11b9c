"""The longest request there can be: 2^31 - 16 keys (the table's row has no room for more), every page of it the same one, so that the
cache is small.  Counts, tiles and the first key behind a tile then come to the end of 32 bits."""
import numpy as np
import pytest
import torch

from tests import _q4_ref as q4
from tests.test_gpu_decode import binding, dev, host, i32  # noqa: F401 (binding is a fixture)

pytestmark = pytest.mark.gpu

PAGE, D = 16, 64
WIDTH = (2 ** 31 - 1) // PAGE
LONGEST = WIDTH * PAGE


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("rows", [1, 3, 30, 150])
def test_tree_attn_over_the_longest_request(binding, bits, rows):  # noqa: F811
    """Rows: 1 to 16 in registers, 17 to 128 and more in tiles."""
    rng = np.random.default_rng(rows)
    hq = 3 if rows > 1 else 1                                                  # 9 rows for three tokens
    tokens = max(rows // hq, 1)
    q = dev(rng.standard_normal((tokens, hq, D)) * 0.5)
    out, lse = torch.full((hq, tokens, D), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((hq, tokens), 9.0, device="cuda")
    table = torch.zeros(1, WIDTH, dtype=torch.int32, device="cuda")
    ctx = binding.Context()
    if bits == 4:
        cache = q4.random_cache(rng, 1, 1, PAGE, D, 0.25)
        k, v = (x[0, 0] for x in q4.unpack(cache, PAGE, D))
        ctx.sp_tree_attn_q4(q.transpose(0, 1), torch.tensor(cache).cuda(), table, i32([LONGEST]), i32([0, tokens]), out, lse_out=lse)
    else:
        kd, vd = (dev(rng.standard_normal((1, 1, PAGE, D))) for _ in range(2))
        k, v = (host(x)[0, 0] for x in (kd, vd))
        ctx.sp_tree_attn(q.transpose(0, 1), kd, vd, table, i32([LONGEST]), i32([0, tokens]), out, lse_out=lse)
    torch.cuda.synchronize()
    assert ctx.status() == (0, 0)
    # Sums.  A chain of n additions in 32 bits is off by n * 2^-24 at most where they round and n * 2^-23 where they cut off.  The work is
    # cut into a run for each SM at least, so that a lane adds up LONGEST / 148 keys at most, 16 and more at a time; with 128 and
    # more rows a tile of 128 keys is eight such steps, or the two halves of one each.
    n = LONGEST / 148 / 16
    off = n * 2.0 ** -23
    assert off < 0.12
    for h in range(hq):
        s = host(q)[:, h] @ k.T / D ** 0.5
        for t in range(tokens):
            count = np.full(PAGE, float(WIDTH))
            for key in range(LONGEST - tokens + t + 1, LONGEST):              # of later tokens
                count[key % PAGE] -= 1
            w = count * np.exp(s[t])
            want = (w @ v) / w.sum()
            # P in bf16, 2^-8 of every weight, and the result
            assert np.all(np.abs(host(out)[h, t] - want) <= (2 * off + 2.0 ** -8) * np.abs(v).max() + 2.0 ** -8 * np.abs(want)), (h, t)
            assert abs(float(lse[h, t]) - np.log(w.sum())) <= off + 2.0 ** -11 + 2.0 ** -20 * 25
