"""NaN, infinities and scales at their ends where they count: a NaN among what a query row attends makes that row NaN, and no other, through every
kernel and merge; none of them is ever taken for a row that sees nothing."""
import math

import numpy as np
import pytest
import torch

from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild
from tests.test_gpu_fp8_paged import _attend, _bounds

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


# ------------------------------------------------------------------ attention over E4M3 pages

LENS, PAGE, S_Q = [300, 130, 65, 0, 1], 32, 2
# kernel: dimensions, path, splits that lead to it, policy, type of the queries
KERNELS = {
    "absorb": ((32, 8, 128, 512, 64), "absorb", (-3, 3, 1), B.POLICY_AUTO, torch.bfloat16),
    "pairs": ((128, 8, 128, 512, 64), "absorb", (-14, 9), B.POLICY_AUTO, torch.bfloat16),
    "gqa": ((32, 8, 128, 512, 64), "gqa", (-3, 3, 1), B.POLICY_AUTO, torch.bfloat16),
    "generic_absorb": ((32, 8, 128, 512, 64), "absorb", (-3, 1), B.POLICY_GENERIC, torch.bfloat16),
    "generic_gqa": ((6, 2, 10, 20, 6), "gqa", (3,), B.POLICY_AUTO, torch.float32),
}
RUNS = [(k, s) for k in KERNELS for s in KERNELS[k][2]]


class Attention:
    """A small call over random finite pages; `run` gives (out, lse) of what its tensors hold then."""

    def __init__(self, kernel, splits, seed=5):
        (self.h, self.g, d_h, r_kv, d_r), self.path, _, self.policy, dtype = KERNELS[kernel]
        self.d, self.splits = B.make_dims(self.h, self.g, d_h, r_kv, d_r), splits
        gen = torch.Generator().manual_seed(seed)
        counts = [-(-t // PAGE) for t in LENS]
        n_pages = sum(counts) + 2
        order = torch.randperm(n_pages, generator=gen).tolist()
        self.table = torch.zeros((len(LENS), max(counts)), dtype=torch.int32)
        for i, c in enumerate(counts):
            self.table[i, :c] = torch.tensor([order.pop() for _ in range(c)], dtype=torch.int32)

        def plane(heads, width):
            codes = torch.randint(0, 0x78, (n_pages * PAGE, heads, width), generator=gen, dtype=torch.uint8)
            codes |= torch.randint(0, 2, codes.shape, generator=gen, dtype=torch.uint8) << 7
            return codes.cuda(), torch.exp2(torch.randint(-9, -5, (n_pages, heads), generator=gen).float()).cuda()

        self.q_split, width, self.dv = (r_kv, r_kv + d_r, r_kv) if self.path == "absorb" else (d_h, d_h + d_r, d_h)
        self.planes = [plane(1, width)] if self.path == "absorb" else [plane(self.g, d_h), plane(self.g, d_h), plane(1, d_r)]
        self.q = (torch.randn((len(LENS), S_Q, self.h, width), generator=gen) * 0.1).to(dtype).cuda()
        self.table, self.lens = self.table.cuda(), torch.tensor(LENS, dtype=torch.int32).cuda()

    def row(self, b, t):
        return int(self.table[b, t // PAGE]) * PAGE + t % PAGE

    def run(self, scale=0.08):
        slots, shape = abs(self.splits), (len(LENS), S_Q, self.h)
        o_part = torch.full((shape[0], slots, *shape[1:], self.dv), 5.0, device="cuda")
        lse_part = torch.full((shape[0], slots, *shape[1:]), 5.0, device="cuda")
        out, lse = torch.full((*shape, self.dv), 5.0, dtype=self.q.dtype, device="cuda"), torch.full(shape, 5.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        tail = (self.table, PAGE, self.lens, scale, self.splits, o_part, lse_part, out, lse, status)
        p = self.planes
        B.set_policy(self.policy)
        try:
            if self.path == "absorb":
                B.gqla_decode_absorb_fp8_paged(self.d, self.q, p[0][0][:, 0], p[0][1][:, 0], *tail)
            else:
                B.gqla_decode_gqa_fp8_paged(self.d, self.q, p[0][0], p[1][0], p[2][0][:, 0], p[0][1], p[1][1], p[2][1][:, 0], *tail)
        finally:
            B.set_policy(B.POLICY_AUTO)
        assert int(status) == 0
        return out, lse


def _only(got, clean, rows):
    """out and lse of `rows` (a mask) are NaN, all others what they were."""
    for x, c in zip(got, clean):
        assert bool(x[rows].isnan().all())
        assert torch.equal(x[~rows], c[~rows])


@pytest.mark.parametrize("kernel,splits", RUNS)
@pytest.mark.parametrize("b,t", [(0, 0), (0, 200), (0, 298), (1, 127), (4, 0)])
def test_a_nan_key_makes_its_rows_nan(kernel, splits, b, t):
    """A NaN code in a row that both positions of the step see (the last sequence: its one row is seen by the last position)."""
    a = Attention(kernel, splits)
    clean = a.run()
    assert all(not bool(x.isnan().any()) for x in clean)
    for plane in (0,) if a.path == "absorb" else (0, 2):
        codes = a.planes[plane][0]
        head = codes.shape[1] // 2
        before = codes[a.row(b, t)].clone()
        codes[a.row(b, t), head, -1] = 0x7F
        rows = torch.zeros((len(LENS), S_Q, a.h), dtype=torch.bool, device="cuda")
        of = a.h // codes.shape[1]
        rows[b, 1 if b == 4 else 0:, head * of:(head + 1) * of] = True
        got = a.run()
        if b == 4 and kernel != "generic_absorb" and a.path == "absorb":
            # (a value NaN times a hidden weight of zero: only lse of the position that does not see the row is kept)
            assert torch.equal(got[1][4, 0], clean[1][4, 0]) and bool(got[0][4, 1].isnan().all()) and bool(got[1][4, 1].isnan().all())
            assert torch.equal(got[0][:4], clean[0][:4]) and torch.equal(got[1][:4], clean[1][:4])
        else:
            _only(got, clean, rows)
        codes[a.row(b, t)] = before


@pytest.mark.parametrize("kernel,splits", [r for r in RUNS if "gqa" in r[0]])
def test_a_nan_value_makes_its_column_nan(kernel, splits):
    a = Attention(kernel, splits)
    out, lse = a.run()
    a.planes[1][0][a.row(0, 150), 1, 3] = 0xFF
    got, got_lse = a.run()
    of = a.h // a.g
    assert torch.equal(got_lse, lse) and bool(got[0, :, of:2 * of, 3].isnan().all())
    got[0, :, of:2 * of, 3] = out[0, :, of:2 * of, 3]
    assert torch.equal(got, out)


@pytest.mark.parametrize("kernel,splits", RUNS)
def test_a_nan_in_the_last_row_and_the_position_before(kernel, splits):
    """The step's first position does not see its last row: no NaN reaches lse there, nor any other column of out than the NaN's."""
    a = Attention(kernel, splits)
    out, lse = a.run()
    col = 3
    plane = a.planes[0 if a.path == "absorb" else 1][0]
    plane[a.row(0, LENS[0] - 1), :, col] = 0x7F
    got, got_lse = a.run()
    assert torch.equal(got_lse[:, 0], lse[:, 0]) and torch.equal(got_lse[1:], lse[1:]) and torch.equal(got[1:], out[1:])
    others = torch.arange(a.dv, device="cuda") != col
    assert torch.equal(got[0, 0, :, others], out[0, 0, :, others]) and bool(got[0, 1, :, col].isnan().all())
    assert a.path == "gqa" or bool(got_lse[0, 1].isnan().all())


@pytest.mark.parametrize("kernel,splits", RUNS)
def test_a_nan_query_makes_its_row_nan(kernel, splits):
    a = Attention(kernel, splits)
    clean = a.run()
    rows = torch.zeros((len(LENS), S_Q, a.h), dtype=torch.bool, device="cuda")
    for b, p, head, col in ((0, 0, 0, 0), (0, 1, a.h - 1, -1), (1, 0, a.h // 2, a.q_split), (4, 1, 1, 5), (3, 0, 2, 2), (4, 0, 2, 2)):
        a.q[b, p, head, col] = math.nan
        rows[b, p, head] = b != 3 and (b, p) != (4, 0)  # (those see nothing: zeros and -inf)
    _only(a.run(), clean, rows)


@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("kernel,splits", RUNS)
def test_an_infinite_query_makes_its_row_nan(kernel, splits, value):
    """Whatever the signs of the keys: alone among small elements, among large ones, twice in a row."""
    a = Attention(kernel, splits)
    clean = a.run()
    rows = torch.zeros((len(LENS), S_Q, a.h), dtype=torch.bool, device="cuda")
    for b, p, head, col in ((0, 0, 0, 0), (0, 1, a.h - 1, -1), (0, 1, a.h - 1, 4), (1, 0, a.h // 2, a.q_split), (2, 1, 3, 7), (4, 1, 1, 5),
                            (3, 0, 2, 2), (4, 0, 2, 2)):
        a.q[b, p, head, col] = value
        rows[b, p, head] = b != 3 and (b, p) != (4, 0)
    _only(a.run(), clean, rows)


@pytest.mark.parametrize("kernel,splits", [r for r in RUNS if "generic" not in r[0]])
def test_huge_queries_are_no_infinities(kernel, splits):
    """Rows times a power of two, which the softmax scale takes away again: bit for bit the same."""
    a = Attention(kernel, splits)
    out, lse = a.run()
    a.q = a.q * 2.0 ** 118
    big, big_lse = a.run(0.08 * 2.0 ** -118)
    assert torch.equal(big, out) and torch.equal(big_lse, lse)


@pytest.mark.parametrize("kernel,splits", RUNS)
@pytest.mark.parametrize("zeros", ["first", "last", "most"])
def test_pages_of_the_smallest_scale_beside_ordinary_ones(kernel, splits, zeros):
    """Pages of zeros as an append writes them (scale 2^-40), one of small codes at that scale and one of a large scale: a zero row
    has a score of zero, which counts in full in the sum."""
    a = Attention(kernel, splits)
    for b, t in enumerate(LENS):
        pages = [int(x) for x in a.table[b, :-(-t // PAGE)]]
        empty = {"first": pages[:2], "last": pages[-2:], "most": pages[:3] + pages[5:]}[zeros]
        for codes, scale in a.planes:
            for page in empty:
                codes[page * PAGE:(page + 1) * PAGE] = 0
                scale[page] = 2.0 ** -40
            if len(pages) > 4:
                scale[pages[3]] = 2.0 ** -4
                scale[pages[4]] = 2.0 ** -40
    out, lse = a.run()
    val = [c.cpu().view(torch.float8_e4m3fn).double().numpy() for c, _ in a.planes]
    scl = [s.cpu().double().numpy() for _, s in a.planes]
    heads = 1 if a.path == "absorb" else a.g
    terms = "e5m2" if kernel == "pairs" else "e4m3"
    for b, t in enumerate(LENS):
        at = np.array([a.row(b, i) for i in range(t)], dtype=np.int64)
        if t == 0:
            assert not out[b].any() and bool(lse[b].isneginf().all())
            continue
        pg = at // PAGE
        for j in range(heads):
            per = a.h // heads
            q = a.q[b, :, j * per:(j + 1) * per].cpu().double().numpy().reshape(S_Q * per, -1)
            if a.path == "absorb":
                k, v8, sv = val[0][at, 0] * scl[0][pg, :1], val[0][at, 0, :a.dv], scl[0][pg, 0]
            else:
                k = np.concatenate([val[0][at, j] * scl[0][pg, j][:, None], val[2][at, 0] * scl[2][pg]], axis=1)
                v8, sv = val[1][at, j], scl[1][pg, j]
            x = q @ k.T * 0.08
            limits = [max(0, t - (S_Q - 1 - p)) for p in range(S_Q) for _ in range(per)]
            o, l_ref, p = _attend(q, x, v8, sv, limits)
            # fp32 sums of exact products, and query elements below 2^-15 of the row's largest, off by 2^-19 of it (as in that module)
            width = q.shape[1]
            x_err = 0.08 * float((np.abs(q) @ np.abs(k).T).max() * 2.0 ** -22 * math.sqrt(width)
                                 + 2.0 ** -25 * np.abs(q).max() * np.abs(k).sum(1).max()) + 2.0 ** -21 * max(1.0, np.abs(x).max())
            bound = _bounds(p, sv[None], v8, x_err, torch.finfo(a.q.dtype).eps / 2, terms)
            got = out[b, :, j * per:(j + 1) * per].cpu().double().numpy().reshape(o.shape)
            got_l = lse[b, :, j * per:(j + 1) * per].cpu().double().numpy().reshape(-1)
            assert (np.abs(got - o) <= bound + 1e-30).all(), (b, j, float((np.abs(got - o) / (bound + 1e-30)).max()))
            live = np.isfinite(l_ref)
            assert np.array_equal(np.isfinite(got_l), live)
            # (the kernels take exponents by the hardware's 2^x and logarithm, 2^-22 of a few tens in log2 units)
            assert (np.abs(got_l[live] - l_ref[live]) <= x_err + 2.0 ** -16).all(), (b, j)
