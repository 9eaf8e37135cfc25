"""What the decoder over E4M3 pages refuses before a projection's call would read or write out of bounds, and the layouts of new rows
that it takes."""
import math

import pytest
import torch

from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild
from paper_2605_15250_b200.decoder import GqlaFp8PagedDecoder

pytestmark = pytest.mark.gpu

DIMS = dict(h_q=32, g=8, d_h=128, r_kv=512, d_r=64)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gbuild.build()
    assert torch.cuda.is_available()
    B.lib()


def _decoder(expanded, lens=(3, 2)):
    gen = torch.Generator().manual_seed(2)
    w = [(torch.randn((8, 512, 128), generator=gen) / math.sqrt(512)).bfloat16().cuda() for _ in range(2)]
    return GqlaFp8PagedDecoder(**DIMS, w_uk=w[0], w_uv=w[1], n_pages=4, page_size=16, block_table=torch.arange(4, dtype=torch.int32).view(2, 2).cuda(),
                               seqlens=torch.tensor(lens, dtype=torch.int32, device="cuda"), scale=0.07,
                               rope=torch.randn((32, 64), generator=gen).cuda(), expanded=expanded)


def _x(*shape, dtype=torch.bfloat16):
    return torch.ones(shape, dtype=dtype, device="cuda")


def test_new_rows_of_another_type_or_width_are_refused():
    dec, start = _decoder(True), torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    for c in (_x(5, 512, dtype=torch.float32), _x(5, 1024, dtype=torch.float32)[:, :512], _x(5, 256), _x(5, 1024)[:, :256], _x(5, 1024),
              _x(5, 512).cpu(), _x(5, 4, 128)):
        with pytest.raises(B.GqlaError, match="c: expected"):
            dec.append_expanded(c, _x(5, 64), start)
    assert not dec.k_c8.any()


def test_queries_of_another_type_or_shape_are_refused():
    dec = _decoder(False)
    good = (_x(2, 1, 32, 128), _x(2, 1, 32, 64))
    dec.absorb_step(*good)
    for i, q in ((0, good[0].float()), (1, good[1].float()), (0, _x(2, 1, 32, 64)), (1, _x(2, 1, 32, 128)), (0, _x(2, 1, 16, 128)),
                 (0, _x(2, 2, 32, 128)), (1, _x(2, 2, 32, 64)), (0, _x(3, 1, 32, 128)), (1, _x(1, 1, 32, 64)), (0, _x(2, 32, 128)),
                 (0, good[0].cpu())):
        args = list(good)
        args[i] = q
        with pytest.raises(B.GqlaError, match="expected"):
            dec.absorb_step(*args)


def test_new_rows_of_any_layout():
    """Dense rows, rows of wider ones, every other column: the same planes."""
    start = torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(4)
    c, k_r = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((5, 512), (5, 64)))
    wide, apart = _x(5, 1200), _x(5, 1024)
    wide[:, 8:520], apart[:, ::2] = c, c
    want = None
    for rows in (c, wide[:, 8:520], apart[:, ::2]):
        dec = _decoder(True)
        dec.append_expanded(rows, k_r, start)
        dec.check_status()
        got = (dec.k_c8, dec.v8, dec.k_r8, dec.k_scale, dec.v_scale, dec.r_scale)
        assert got[0].any() and (want is None or all(torch.equal(a, b) for a, b in zip(got, want)))
        want = got
