"""New rows behind the last sequence's (a batch padded to a fixed number of rows): left out of the cache, the scales and the queries."""
import numpy as np
import pytest
import torch

from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild

pytestmark = pytest.mark.gpu

PAGE, H_Q, G, D_H, R_KV, D_R = 16, 32, 8, 128, 512, 64
# lengths, new rows, padding rows; the last sequence ends with its page, so that padding rows would start the next one
BATCHES = {"step": ([20, 33, 32], [1, 1, 1], 5), "prompts": ([70, 5, 64], [70, 5, 64], 40), "no rows": ([20, 32], [0, 0], 3),
           "padding sequences": ([20, 32, 0, 0], [1, 2, 0, 0], 4), "one row behind": ([31, 48], [2, 48], 1)}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gbuild.build()
    assert torch.cuda.is_available()
    B.lib()


@pytest.mark.parametrize("batch", sorted(BATCHES))
@pytest.mark.parametrize("kind", ["packed", "paged", "latent", "planes"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_behind_the_last_sequence_are_left_alone(kind, batch, dtype):
    lens, new, pad = BATCHES[batch]
    n, d = sum(new), B.make_dims(H_Q, G, D_H, R_KV, D_R)
    gen = torch.Generator(device="cuda").manual_seed(3)
    max_pages = -(-max(lens) // PAGE) + 4
    n_pages = len(lens) * max_pages
    # entries behind a sequence's end name pages of the pool that are nobody's
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).view(len(lens), max_pages).to(torch.int32).cuda()
    rope = torch.randn((256, D_R), generator=gen, device="cuda")
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    c, k_c, v, k_r, q = (normal(n + pad, *s) for s in ((R_KV,), (G, D_H), (G, D_H), (D_R,), (H_Q, D_R)))
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    seq_start = torch.tensor([128 * i for i in range(len(lens))], dtype=torch.int64, device="cuda")
    results = []
    for rows in (n, n + pad):
        q_out = torch.full((n + pad, H_Q, D_R), 9.0, dtype=dtype, device="cuda")
        bytes_ = lambda *s: torch.full(s, 0x31, dtype=torch.uint8, device="cuda")  # noqa: E731
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        step = (start, sl, rope, "pairs")
        turned = (q[:rows], q_out[:rows], status)
        if kind in ("packed", "paged"):
            cache = torch.full((n_pages * PAGE, R_KV + D_R), 3.0, dtype=dtype, device="cuda")
            where = (seq_start, None, 0) if kind == "packed" else (None, table, PAGE)
            B.gqla_append_rope(d, c[:rows], k_r[:rows], *step, cache, *where, *turned)
            state = [cache]
        elif kind == "latent":
            state = [bytes_(n_pages * PAGE, R_KV + D_R), torch.full((n_pages,), 0.5, device="cuda")]
            B.gqla_append_rope_fp8(d, c[:rows], k_r[:rows], *step, *state, table, PAGE, *turned)
        else:
            state = [bytes_(n_pages * PAGE, G, D_H), bytes_(n_pages * PAGE, G, D_H), bytes_(n_pages * PAGE, D_R),
                     *(torch.full(s, 0.5, device="cuda") for s in ((n_pages, G), (n_pages, G), (n_pages,)))]
            B.gqla_append_planes_fp8(d, k_c[:rows], v[:rows], k_r[:rows], *step, *state, table, PAGE, *turned)
        assert int(status) == 0
        results.append((*state, q_out))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert bool((results[1][-1][n:] == 9.0).all())
