"""Where the pieces of attention over E4M3 pages lie: lse of every split slot against the plan that the header documents."""
import math

import numpy as np
import pytest
import torch

from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild

pytestmark = pytest.mark.gpu

PAGE = 64
CANON, LLAMA, MANY = (128, 8, 128, 512, 64), (32, 8, 128, 512, 64), (40, 1, 128, 512, 64)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gbuild.build()
    assert torch.cuda.is_available()
    B.lib()


def _documented(lens, slots, workers, path, rows):
    """Row ranges [sequence][slot] by the header's words."""
    tiles = [-(-t // 128) for t in lens]
    share = max(-(-sum(tiles) // workers), -(-max(tiles) // (slots - 1)), 1)
    slack = 3 if path == "absorb" and rows <= 64 else 6
    if len(lens) <= workers < 2 * len(lens) and share > 1 and max(tiles) <= share + slack:
        return [[(0, t)] + [(0, 0)] * (slots - 1) for t in lens]
    return B.gqla_balanced_plan(lens, slots, workers)[0]


def _lens(kind, batch):
    rng = np.random.default_rng(batch)
    if kind == "even":
        return [int(t) for t in rng.integers(400, 640, size=batch)]
    lens = [int(t) for t in rng.integers(0, 500, size=batch)]
    lens[batch // 2] = 6000 if kind == "long" else 1100
    return lens


@pytest.mark.parametrize("path,dims,s_q,batch,kind,slots", [
    # more than 64 rows of the absorb path: no more pieces than CTAs for them, or on pairs
    ("absorb", CANON, 1, 20, "ragged", 2), ("absorb", CANON, 1, 30, "ragged", 2), ("absorb", CANON, 1, 30, "even", 2),
    ("absorb", CANON, 1, 9, "ragged", 5), ("absorb", CANON, 2, 10, "even", 2), ("absorb", MANY, 2, 25, "ragged", 2),
    ("absorb", CANON, 1, 1, "long", 12), ("absorb", CANON, 1, 36, "even", 2), ("absorb", CANON, 1, 60, "even", 2),
    ("absorb", CANON, 1, 60, "even", 5), ("absorb", CANON, 1, 60, "long", 5), ("absorb", CANON, 1, 80, "ragged", 3),
    # the others
    ("absorb", LLAMA, 1, 110, "even", 3), ("absorb", LLAMA, 1, 110, "ragged", 2), ("absorb", LLAMA, 1, 110, "long", 4),
    ("absorb", LLAMA, 2, 30, "ragged", 2), ("gqa", LLAMA, 1, 14, "even", 3), ("gqa", LLAMA, 1, 14, "long", 6), ("gqa", CANON, 2, 5, "ragged", 9)])
def test_pieces_lie_where_the_plan_says(path, dims, s_q, batch, kind, slots):
    h_q, g, d_h, r_kv, d_r = dims
    d, lens = B.make_dims(*dims), _lens(kind, batch)
    workers = B.gqla_fp8_paged_workers(d, torch.bfloat16, s_q, PAGE, path)
    assert workers > 0
    gen = torch.Generator(device="cuda").manual_seed(batch)
    pages = [-(-t // PAGE) for t in lens]
    n_pages = sum(pages)
    table = torch.zeros((batch, max(pages)), dtype=torch.int32)
    first = np.concatenate([[0], np.cumsum(pages)])
    for i, n in enumerate(pages):
        table[i, :n] = torch.arange(first[i], first[i] + n)
    codes = lambda *s: torch.randint(0, 0x60, (n_pages * PAGE, *s), generator=gen, dtype=torch.uint8, device="cuda")  # noqa: E731
    one = lambda *s: torch.full((n_pages, *s), 2.0 ** -4, device="cuda")  # noqa: E731
    width, dv = (r_kv + d_r, r_kv) if path == "absorb" else (d_h + d_r, d_h)
    q = (torch.randn((batch, s_q, h_q, width), generator=gen, device="cuda") * 0.05).bfloat16()
    o_part = torch.empty((batch, slots, s_q, h_q, dv), device="cuda")
    lse_part = torch.full((batch, slots, s_q, h_q), math.nan, device="cuda")
    tail = (table.cuda(), PAGE, torch.tensor(lens, dtype=torch.int32, device="cuda"), 0.1, -slots, o_part, lse_part)
    if path == "absorb":
        cache = codes(width)
        B.gqla_decode_absorb_fp8_paged(d, q, cache, one(), *tail)
        keys = cache.view(torch.float8_e4m3fn).double()[:, None].expand(-1, g, -1) * 2.0 ** -4
    else:
        k_c, v, k_r = codes(g, d_h), codes(g, d_h), codes(d_r)
        B.gqla_decode_gqa_fp8_paged(d, q, k_c, v, k_r, one(g), one(g), one(), *tail)
        keys = torch.cat([k_c.view(torch.float8_e4m3fn).double(), k_r.view(torch.float8_e4m3fn).double()[:, None].expand(-1, g, -1)], -1) * 2.0 ** -4
    plan = _documented(lens, slots, workers, path, s_q * h_q)
    used = 0
    for b, t in enumerate(lens):
        at = int(first[b]) * PAGE
        x = torch.einsum("sgpw,tgw->sgpt", q[b].double().view(s_q, g, -1, width), keys[at:at + t]).reshape(s_q, h_q, t) * 0.1
        for p in range(s_q):
            seen = max(0, t - (s_q - 1 - p))
            for k, (lo, hi) in enumerate(plan[b]):
                hi = min(hi, seen)
                got = lse_part[b, k, p].double()
                if hi <= lo:
                    assert bool(got.isneginf().all()), (b, k, p)
                    continue
                used += 1
                # fp32 sums of at most 576 exact products of size 2^-4 * 60 * 0.2 each, far below a step of the sum of exponentials
                assert float((got - torch.logsumexp(x[p, :, lo:hi], -1)).abs().max()) <= 1e-4, (b, k, p)
    assert used >= batch // 2
