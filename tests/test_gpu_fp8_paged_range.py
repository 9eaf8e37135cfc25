"""Ends of the documented range of the append calls and of attention over E4M3 pages: hundreds and thousands of query positions, and
layers without a rotated part."""
import numpy as np
import pytest
import torch

from oracle import gqla_oracle as O
from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild
from tests.test_gpu_fp8_paged import CANON, LLAMA, _check_attention, _dev, _f64, _few_bits, _pages, _same_codes, _starts, _table

pytestmark = pytest.mark.gpu

NO_ROPE = dict(h_q=6, g=2, d_h=16, r_kv=32, d_r=0)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gbuild.build()
    assert torch.cuda.is_available()
    B.lib()


@pytest.mark.parametrize("path,dims", [("absorb", LLAMA), ("gqa", LLAMA), ("gqa", CANON), ("absorb", CANON)])
@pytest.mark.parametrize("splits", [-2, 1, 3])
def test_a_chunk_of_a_prompt(path, dims, splits):
    """As many query positions as a chunk has, over a cache that is longer, as long and shorter."""
    _check_attention(path, dims, [500, 130, 129, 7, 0], 130, 64, splits)


@pytest.mark.parametrize("path", ["absorb", "gqa"])
@pytest.mark.parametrize("s_q", [4096, 4097])
def test_thousands_of_query_positions(path, s_q):
    """The most that the tensor-core kernels take, and one more; nearly all of them see nothing."""
    _check_attention(path, LLAMA, [10, 150], s_q, 32, -2)


@pytest.mark.parametrize("path", ["absorb", "gqa"])
@pytest.mark.parametrize("splits", [-3, 2])
def test_attention_without_a_rotated_part(path, splits):
    _check_attention(path, NO_ROPE, [90, 0, 1, 33], 2, 16, splits, dtype=torch.float32)
    _check_attention(path, NO_ROPE, [90, 0, 1, 33], 2, 24, splits)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,new", [([33, 64, 65], [1, 1, 1]), ([100, 20, 64], [100, 3, 64])])
def test_appends_without_a_rotated_part(dtype, lens, new):
    rng = np.random.default_rng(3)
    page, n, d = 16, sum(new), B.make_dims(**NO_ROPE)
    table, n_pages = _table(rng, lens, page)
    none = lambda *s: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    step = (_dev(_starts(new)), _dev(np.array(lens, np.int32)), torch.empty((0, 0), device="cuda"), "pairs")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, k_c, v = (_few_bits(rng, (n, *s), dtype) for s in ((32,), (2, 16), (2, 16)))
    cache = torch.full((n_pages * page, 32), 3.0, dtype=dtype, device="cuda")
    B.gqla_append_rope(d, c.cuda(), none(n, 0), *step, cache, None, _dev(table), page, none(n, 6, 0), none(n, 6, 0), status)
    want = torch.full(cache.shape, 3.0, dtype=dtype)
    for i, (b, t) in enumerate(O.new_row_places(_starts(new), lens)):
        want[int(table[b, t // page]) * page + t % page] = c[i]
    assert torch.equal(cache.cpu(), want)
    planes = [_pages(rng, n_pages, page, h, w) for h, w in ((1, 32), (2, 16), (2, 16))]
    dev = [(_dev(codes), _dev(scale)) for codes, scale in planes]
    B.gqla_append_rope_fp8(d, c.cuda(), none(n, 0), *step, dev[0][0].view(-1, 32), dev[0][1].view(-1), _dev(table), page, status_word=status)
    r8, r_scale = torch.empty((n_pages * page, 0), dtype=torch.uint8, device="cuda"), torch.ones(n_pages, device="cuda")
    B.gqla_append_planes_fp8(d, k_c.cuda(), v.cuda(), none(n, 0), *step, dev[1][0], dev[2][0], r8, dev[1][1], dev[2][1], r_scale, _dev(table),
                             page, status_word=status)
    for (codes, scale), (codes0, scale0), rows in zip(dev, planes, (_f64(c)[:, None], _f64(k_c), _f64(v))):
        want_codes, want_scale = O.append_pages_e4m3(rows, codes0, scale0, _starts(new), lens, table, page)
        assert np.array_equal(scale.cpu().numpy(), want_scale) and _same_codes(codes.cpu().numpy(), want_codes).all()
    assert int(status) == 0 and bool((r_scale == 1).all())
