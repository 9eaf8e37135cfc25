"""NaN and infinities where they count: a NaN among what a query row attends makes that row NaN, and no other, through every
kernel and merge; none of them is ever taken for a row that sees nothing."""
import math

import numpy as np
import pytest
import torch

from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gbuild.build()
    assert torch.cuda.is_available()
    B.lib()
    yield
    B.set_policy(B.POLICY_AUTO)


def _partials(rng, batch, slots, s_q, h_q, width):
    """Partials of which row 0 has a NaN slot among live ones, row 1 one among empty ones, row 2 no live slot, row 3 the partials
    of an empty slot that hold NaN."""
    o = rng.standard_normal((batch, slots, s_q, h_q, width)).astype(np.float32)
    lse = rng.standard_normal((batch, slots, s_q, h_q)).astype(np.float32)
    flat_o, flat_l = (x.reshape(batch, slots, s_q * h_q, -1) for x in (o, lse))
    at = slots // 2
    flat_l[:, at, 0] = np.nan
    flat_o[:, at, 0] = np.nan
    flat_l[:, :, 1:3] = -np.inf
    flat_o[:, :, 1:3] = np.nan
    flat_l[:, at, 1] = np.nan
    flat_l[:, at, 3] = -np.inf
    flat_o[:, at, 3] = np.nan
    return torch.from_numpy(o).cuda(), torch.from_numpy(lse).cuda()


def _merged(o, lse):
    """The merge in 64 bits; slots whose lse is -inf are empty."""
    o, lse = o.double(), lse.double()
    top = lse.nan_to_num(nan=-math.inf, neginf=-math.inf).amax(1, keepdim=True)
    w = torch.exp(lse - torch.where(top > -math.inf, top, 0.0))
    den = w.sum(1)
    out = torch.where((w != 0)[..., None], w[..., None] * o, 0.0).sum(1) / torch.where(den == 0, 1.0, den)[..., None]
    return out, torch.where(den == 0, -math.inf, top[:, 0] + den.log())


def _same(got, want, bound):
    """Rows that are NaN are NaN in full, the others within bound."""
    got = got.double()
    dead = want.isnan()
    assert torch.equal(got.isnan(), dead)
    assert bool(((got - want).abs()[~dead] <= bound).all())


# every form of the merge: columns per thread, thread groups, more slots than are staged, the odd widths' kernel
@pytest.mark.parametrize("batch,slots,h_q,width", [(2, 2, 8, 128), (3, 5, 8, 512), (2, 40, 8, 512), (400, 3, 32, 512), (60, 3, 32, 512),
                                                   (2, 1100, 4, 128), (2, 4, 6, 10), (2, 9, 6, 7), (2, 1, 8, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_merge_passes_on_a_nan(batch, slots, h_q, width, dtype):
    o_part, lse_part = _partials(np.random.default_rng(1), batch, slots, 1, h_q, width)
    out = torch.full((batch, 1, h_q, width), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((batch, 1, h_q), 7.0, device="cuda")
    B.gqla_combine_splits(o_part, lse_part, out, lse)
    want, want_lse = _merged(o_part, lse_part)
    rows = want_lse[:, 0]
    assert bool(rows[:, :2].isnan().all()) and bool(rows[:, 2].isneginf().all()) and not bool(rows[:, 4:].isnan().any())
    # weights and sums of at most 1100 slots in fp32 (a few 2^-24 each, relative to values up to 5), half a step of the type
    _same(out, want, 6 * (torch.finfo(dtype).eps / 2 + 2.0 ** -18))
    live = torch.isfinite(want_lse)
    assert torch.equal(lse.isneginf(), want_lse.isneginf()) and torch.equal(lse.isnan(), want_lse.isnan())
    assert bool(((lse.double() - want_lse).abs()[live] <= 2.0 ** -18).all())


@pytest.mark.parametrize("dims,dtype,slots", [((32, 8, 128, 512, 64), torch.bfloat16, 3), ((128, 8, 128, 512, 64), torch.bfloat16, 40),
                                              ((8, 2, 48, 96, 16), torch.bfloat16, 4), ((8, 2, 48, 96, 16), torch.float32, 4)])
def test_merge_with_up_projection_passes_on_a_nan(dims, dtype, slots):
    h_q, g, d_h, r_kv, _ = dims
    o_part, lse_part = _partials(np.random.default_rng(2), 3, slots, 1, h_q, r_kv)
    gen = torch.Generator().manual_seed(3)
    w_uv = (torch.randn((g, r_kv, d_h), generator=gen) / math.sqrt(r_kv)).to(dtype).cuda()
    o = torch.full((3, 1, h_q, d_h), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((3, 1, h_q), 7.0, device="cuda")
    B.gqla_combine_up_proj(B.make_dims(*dims), o_part, lse_part, w_uv, o, lse)
    o_hat, want_lse = _merged(o_part, lse_part)
    up = lambda x, w: torch.einsum("bsgpr,grd->bsgpd", x.view(3, 1, g, h_q // g, r_kv), w).reshape(3, 1, h_q, d_h)  # noqa: E731
    want = up(o_hat, w_uv.double())
    # the merged row and the output are rounded to the type, half a step each; sums in fp32
    eps = torch.finfo(dtype).eps / 2 + 2.0 ** -18
    bound = eps * (up(o_hat.abs(), w_uv.double().abs()) * (1 + eps) + want.abs())
    _same(o, want, bound[~want.isnan()])
    assert torch.equal(lse.isneginf(), want_lse.isneginf()) and torch.equal(lse.isnan(), want_lse.isnan())
