"""E4M3 pages with a scale per page and head: the append calls (rotation, scales, codes, what they leave alone) and the
attention of both paths over what they write, against the oracle in 64 bits; a run of them as a server makes it."""
import math

import numpy as np
import pytest
import torch

from oracle import gqla_oracle as O
from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild
from paper_2605_15250_b200.decoder import GqlaDecoder, GqlaFp8PagedDecoder
from tests.parity_util import Canaried

pytestmark = pytest.mark.gpu

CANON = dict(h_q=128, g=8, d_h=128, r_kv=512, d_r=64)
LLAMA = dict(h_q=32, g=8, d_h=128, r_kv=512, d_r=64)
TINY = dict(h_q=6, g=2, d_h=10, r_kv=20, d_r=6)
UNEVEN = dict(h_q=8, g=2, d_h=48, r_kv=96, d_r=16)  # vectors of eight that do not divide a block's threads


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gbuild.build()
    assert torch.cuda.is_available()
    B.lib()
    yield
    B.set_policy(B.POLICY_AUTO)


@pytest.fixture
def rng():
    return np.random.default_rng(5)


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def _f64(t):
    return t.detach().cpu().double().numpy()


def _table(rng, lens, page, spare=3):
    """A shuffled pool: block table [B, max_pages] and the number of pages; entries behind a sequence's end name no page."""
    counts = [-(-t // page) for t in lens]
    n = sum(counts) + spare
    order = rng.permutation(n)
    table = np.full((len(lens), max(max(counts), 1)), -7, dtype=np.int32)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = order[at:at + c]
        at += c
    return table, n


def _angles(n, d_r):
    freq = 10000.0 ** (-np.arange(0, d_r, 2) / d_r)
    a = np.arange(n)[:, None] * freq
    return np.concatenate([np.cos(a), np.sin(a)], axis=1).astype(np.float32)


def _exact_turns(rng, n, d_r):
    """Cosines and sines from multiples of 1/4: every product and sum with few-bit rows is exact in fp32, so that no rounding
    stands between a code and its definition."""
    return (rng.integers(-4, 5, size=(n, d_r)) / 4.0).astype(np.float32)


def _starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def _few_bits(rng, shape, dtype):
    """Random rows of magnitudes 2^-6 .. 2^6 with five significant bits."""
    return torch.from_numpy(np.ldexp(rng.integers(-31, 32, size=shape), rng.integers(-10, 3, size=shape)).astype(np.float32)).to(dtype)


# ------------------------------------------------------------------ appending

LENGTHS = {  # lengths and new rows: a step, prompts, both, nothing new, sequences shorter than their new rows, one row
    "step": ([33, 64, 65, 1, 200], [1, 1, 1, 1, 1]),
    "drafts": ([40, 64, 17, 129], [3, 3, 3, 3]),
    "prompts": ([100, 1, 64, 257], [100, 1, 64, 257]),
    "mixed": ([70, 150, 16, 90], [0, 150, 2, 40]),
    "short": ([2, 0, 5, 30], [4, 3, 5, 1]),
    "one": ([777], [1]),
    "first": ([1], [1]),
}


@pytest.mark.parametrize("style", ["pairs", "halves"])
@pytest.mark.parametrize("case", sorted(LENGTHS))
@pytest.mark.parametrize("dims,dtype,paged", [(CANON, torch.bfloat16, True), (CANON, torch.float32, False), (TINY, torch.float32, True),
                                              (TINY, torch.bfloat16, False), (UNEVEN, torch.bfloat16, True)])
def test_append_rope_rows_and_queries(rng, dims, dtype, paged, case, style):
    lens, new = LENGTHS[case]
    d, n, page = B.make_dims(**dims), sum(new), 24
    table, n_pages = _table(rng, lens, page)
    starts = np.cumsum([0] + [t + 5 for t in lens])[:-1]
    rows = n_pages * page if paged else int(sum(lens)) + 5 * len(lens) + 7
    c, k_r, q = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dtype)
                 for s in ((n, dims["r_kv"]), (n, dims["d_r"]), (n, dims["h_q"], dims["d_r"])))
    rope = _angles(max(lens) + 1, dims["d_r"])
    width = dims["r_kv"] + dims["d_r"]
    cache = Canaried((rows, width), dtype)
    before = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).to(dtype)
    cache.t.copy_(before)
    q_out = Canaried(q.shape, dtype)
    q_out.t.fill_(9.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.gqla_append_rope(d, c.cuda(), k_r.cuda(), _dev(_starts(new)), _dev(np.array(lens, np.int32)), _dev(rope), style, cache.t,
                       None if paged else _dev(starts.astype(np.int64)), _dev(table) if paged else None, page if paged else 0,
                       q.cuda(), q_out.t, status)
    places = O.new_row_places(_starts(new), lens)
    kept = [i for i, (_, t) in enumerate(places) if t >= 0]
    pos = [places[i][1] for i in kept]
    want = _f64(before).copy()
    at = [int(table[b, t // page]) * page + t % page if paged else int(starts[b]) + t for b, t in (places[i] for i in kept)]
    turned = O.rope_turn(_f64(k_r)[kept], pos, rope, style)
    got = _f64(cache.t)
    for i, a in zip(kept, at):
        assert np.array_equal(got[a, :dims["r_kv"]], _f64(c)[i])
        want[a] = got[a]
    assert np.array_equal(got, want), "a row that is not new was written"
    # two fp32 products and a sum, then one rounding to the storage type: half a step of it and a few of fp32's, of the pair's size
    eps = torch.finfo(dtype).eps / 2 + 3 * 2.0 ** -24
    size = np.abs(_f64(k_r)[kept]).max(initial=0.0) * 2 ** 0.5
    assert np.abs(got[at, dims["r_kv"]:] - turned).max(initial=0.0) <= eps * size
    q_want = O.rope_turn(_f64(q)[kept], pos, rope, style)
    q_got = _f64(q_out.t)
    assert np.abs(q_got[kept] - q_want).max(initial=0.0) <= eps * np.abs(_f64(q)).max(initial=0.0) * 2 ** 0.5
    skipped = [i for i in range(n) if i not in kept]
    assert (q_got[skipped] == 9.0).all()
    cache.check("cache")
    q_out.check("q_out")
    assert int(status) == 0


def test_append_rope_strided_rows_and_queries_in_place(rng):
    """Rows that are views of wider ones, and the queries' rotated part turned where it lies."""
    d, n = B.make_dims(**CANON), 5
    wide = torch.from_numpy(rng.standard_normal((n, 1536 + 600)).astype(np.float32)).bfloat16().cuda()
    c, k_r = wide[:, 8:520], wide[:, 528:592]
    q = torch.from_numpy(rng.standard_normal((n, 128, 192)).astype(np.float32)).bfloat16().cuda()
    head, tail = q[..., :128].clone(), q[..., 128:].clone()
    pool = torch.zeros((64, 640), dtype=torch.bfloat16, device="cuda")
    table, rope = torch.tensor([[1]], dtype=torch.int32, device="cuda"), _angles(40, 64)
    lens = torch.tensor([30], dtype=torch.int32, device="cuda")
    B.gqla_append_rope(d, c, k_r, torch.tensor([0, n], dtype=torch.int32, device="cuda"), lens, _dev(rope), "pairs", pool[:, :576], None,
                       table, 32, q[..., 128:], q[..., 128:])
    pos = list(range(25, 30))
    assert torch.equal(pool[57:62, :512], c) and torch.equal(q[..., :128], head)
    assert not pool[:57].any() and not pool[62:].any() and not pool[:, 576:].any()
    eps = 2.0 ** -8 + 2.0 ** -22
    for got, src in ((pool[57:62, 512:576], k_r), (q[..., 128:], tail)):
        assert np.abs(_f64(got) - O.rope_turn(_f64(src), pos, rope, "pairs")).max() <= eps * float(src.float().abs().max()) * 2 ** 0.5


def _pages(rng, n_pages, page, heads, width):
    """Pages in use: random codes (no NaN) and power-of-two scales."""
    codes = rng.integers(0, 256, size=(n_pages * page, heads, width)).astype(np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x3A
    return codes, (2.0 ** rng.integers(-8, -1, size=(n_pages, heads))).astype(np.float32)


def _same_codes(got, want):
    return (got == want) | (((got & 0x7F) == 0) & ((want & 0x7F) == 0))


@pytest.mark.parametrize("style", ["pairs", "halves"])
@pytest.mark.parametrize("page", [16, 24, 64, 256])
@pytest.mark.parametrize("case", sorted(LENGTHS))
@pytest.mark.parametrize("dims,dtype", [(LLAMA, torch.bfloat16), (LLAMA, torch.float32), (TINY, torch.bfloat16), (TINY, torch.float32),
                                        (UNEVEN, torch.bfloat16)])
def test_append_fp8_codes_and_scales_bit_for_bit(rng, dims, dtype, case, page, style):
    lens, new = LENGTHS[case]
    d, n = B.make_dims(**dims), sum(new)
    table, n_pages = _table(rng, lens, page)
    rope = _exact_turns(rng, max(lens) + 1, dims["d_r"])
    args = (_dev(_starts(new)), _dev(np.array(lens, np.int32)), _dev(rope), style)
    places = O.new_row_places(_starts(new), lens)
    pos = [max(t, 0) for _, t in places]
    c, k_r = _few_bits(rng, (n, dims["r_kv"]), dtype), _few_bits(rng, (n, dims["d_r"]), dtype)
    turned = O.rope_turn(_f64(k_r), pos, rope, style)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    where = (_dev(table), page)

    def compare(name, cache, scale, rows, codes0, scale0):
        want_codes, want_scale = O.append_pages_e4m3(rows, codes0, scale0, _starts(new), lens, table, page)
        assert np.array_equal(scale.t.cpu().numpy().reshape(scale0.shape), want_scale), name
        same = _same_codes(cache.t.cpu().numpy().reshape(codes0.shape), want_codes)
        assert same.all(), (name, np.argwhere(~same)[:4])
        cache.check(name)
        scale.check(name)

    def buffers(codes0, scale0, shape, scale_shape):
        cache, scale = Canaried(shape, torch.uint8), Canaried(scale_shape, torch.float32)
        cache.t.copy_(torch.from_numpy(codes0.reshape(shape)))
        scale.t.copy_(torch.from_numpy(scale0.reshape(scale_shape)))
        return cache, scale

    # latent pages: [c ; rotated k_r] under one scale
    width = dims["r_kv"] + dims["d_r"]
    codes0, scale0 = _pages(rng, n_pages, page, 1, width)
    cache, scale = buffers(codes0, scale0, (n_pages * page, width), (n_pages,))
    B.gqla_append_rope_fp8(d, c.cuda(), k_r.cuda(), *args, cache.t, scale.t, *where, status_word=status)
    compare("latent", cache, scale, np.concatenate([_f64(c), turned], axis=1)[:, None], codes0, scale0)
    # planes: a scale per page and group
    g, d_h = dims["g"], dims["d_h"]
    k_c, v = _few_bits(rng, (n, g, d_h), dtype), _few_bits(rng, (n, g, d_h), dtype)
    planes = [_pages(rng, n_pages, page, h, w) for h, w in ((g, d_h), (g, d_h), (1, dims["d_r"]))]
    bufs = [buffers(*p, (n_pages * page, g, d_h), (n_pages, g)) for p in planes[:2]]
    bufs.append(buffers(*planes[2], (n_pages * page, dims["d_r"]), (n_pages,)))
    B.gqla_append_planes_fp8(d, k_c.cuda(), v.cuda(), k_r.cuda(), *args, *(b[0].t for b in bufs), *(b[1].t for b in bufs), *where,
                             status_word=status)
    for name, buf, rows, p in zip(("k_c", "v", "k_r"), bufs, (_f64(k_c), _f64(v), turned[:, None]), planes):
        compare(name, *buf, rows, *p)
    assert int(status) == 0


def test_append_fp8_special_values(rng):
    """Zeros, infinities, NaN, subnormal and huge rows; a page of zeros takes the smallest scale, and a later row of ordinary size
    gets the scale that it needs."""
    d, page = B.make_dims(**LLAMA), 16
    table = np.array([[2], [0], [1], [3]], dtype=np.int32)
    c = np.zeros((4, 512), np.float32)
    c[1, :4] = [np.inf, -np.inf, np.nan, 3.0]
    c[2, :3] = [1e-30, -1e-38, 2e-12]
    c[3, :2] = [3e38, -1.5]
    codes = Canaried((5 * page, 576), torch.uint8)
    codes.t.fill_(0x7F)
    scale = torch.full((5,), 3.0, device="cuda")
    zeros = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    rope = _dev(_angles(4, 64))
    one = torch.ones(4, dtype=torch.int32, device="cuda")
    start = torch.arange(5, dtype=torch.int32, device="cuda")
    B.gqla_append_rope_fp8(d, _dev(c, torch.bfloat16), zeros, start, one, rope, "pairs", codes.t, scale, _dev(table), page)
    s = scale.cpu().tolist()
    huge = float(torch.tensor(3e38).bfloat16())
    assert s == [O.pow2_scale(3.0), 2.0 ** -40, 2.0 ** -40, O.pow2_scale(huge), 3.0]
    got = codes.t.cpu().numpy()
    assert not got[2 * page].any() and list(got[0, :4] & 0x7F) == [0x7E, 0x7E, 0x7F, int(O.e4m3_encode(np.array([3.0 / s[0]]))[0])]
    assert got[0, 1] == 0xFE
    b16 = _f64(torch.from_numpy(c).bfloat16())
    assert _same_codes(got[page, :3], O.e4m3_encode(b16[2, :3] / s[1])).all()
    assert _same_codes(got[3 * page, :2], O.e4m3_encode(b16[3, :2] / s[3])).all()
    assert (got[1:page] == 0x7F).all() and (got[4 * page:] == 0x7F).all()
    # the second row of the page of zeros
    two = torch.tensor([2, 2, 2, 2], dtype=torch.int32, device="cuda")
    B.gqla_append_rope_fp8(d, torch.full((4, 512), 0.3, dtype=torch.bfloat16, device="cuda"), zeros, start, two, rope, "pairs", codes.t,
                           scale, _dev(table), page)
    want = O.pow2_scale(float(torch.tensor(0.3).bfloat16()))
    assert scale.cpu().tolist() == [s[0], want, want, s[3], 3.0]
    codes.check("codes")


def test_append_keeps_a_larger_scale_of_the_callers(rng):
    """A page whose older rows came with a scale of another kind: it stays while the new rows fit, and they are coded with it."""
    page, s_old = 16, 0.3
    codes = Canaried((page, 576), torch.uint8)
    codes.t.fill_(0x31)
    scale = torch.full((1,), s_old, device="cuda")
    x = rng.standard_normal((3, 512)).astype(np.float32)
    c = _dev(x, torch.bfloat16)
    B.gqla_append_rope_fp8(B.make_dims(**LLAMA), c, torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda"), _dev(_starts([3])),
                           torch.tensor([8], dtype=torch.int32, device="cuda"), _dev(_angles(8, 64)), "pairs", codes.t, scale,
                           torch.zeros((1, 1), dtype=torch.int32, device="cuda"), page)
    codes.check("codes")
    assert float(scale) == float(np.float32(s_old)) and (codes.t[:5] == 0x31).all() and (codes.t[8:] == 0x31).all()
    got = O.e4m3_decode(codes.t[5:8].cpu().numpy())[:, :512] * float(scale)
    # half a step of E4M3 (2^-4, or 2^-10 of the scale for the smallest codes), and two roundings of 1 / s and the product before it
    assert (np.abs(got - _f64(c)) <= np.abs(_f64(c)) * (2.0 ** -4 + 2.0 ** -22) + 2.0 ** -10 * s_old * 1.001).all()


@pytest.mark.parametrize("kind", ["bf16", "latent", "planes"])
def test_append_leaves_out_what_has_no_place(rng, kind):
    """Positions behind the rotation table or the block table and pages outside the cache are left out and reported; the other
    rows are written."""
    d, page, n_pages = B.make_dims(**LLAMA), 16, 6
    cases = [(dict(rope=20), 1, [2]), (dict(table=[[0, 1], [2, 6], [3, 4]]), 2, [1]), (dict(table=[[0, 1], [2, -1], [3, 4]]), 2, [1]),
             (dict(max_pages=1), 2, [0, 1, 2])]
    for change, code, bad in cases:
        lens = np.array([19, 20, 21] if "rope" in change else [17, 18, 19], np.int32)
        table = np.array(change.get("table", [[0, 1], [2, 5], [3, 4]]), np.int32)[:, :change.get("max_pages", 2)]
        rope = _dev(_angles(change.get("rope", 32), 64))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = (torch.arange(4, dtype=torch.int32, device="cuda"), _dev(lens), rope, "pairs")
        x = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        if kind == "bf16":
            buf = Canaried((n_pages * page, 576), torch.bfloat16)
            buf.t.zero_()
            B.gqla_append_rope(d, x(3, 512), x(3, 64), *args, buf.t, None, _dev(table), page, status_word=status)
        elif kind == "latent":
            buf = Canaried((n_pages * page, 576), torch.uint8)
            buf.t.zero_()
            B.gqla_append_rope_fp8(d, x(3, 512), x(3, 64), *args, buf.t, torch.ones(n_pages, device="cuda"), _dev(table), page,
                                   status_word=status)
        else:
            buf = Canaried((n_pages * page, 8, 128), torch.uint8)
            buf.t.zero_()
            v8, k_r8 = torch.zeros_like(buf.t), torch.zeros((n_pages * page, 64), dtype=torch.uint8, device="cuda")
            s8 = [torch.ones((n_pages, 8), device="cuda") for _ in range(2)] + [torch.ones(n_pages, device="cuda")]
            B.gqla_append_planes_fp8(d, x(3, 8, 128), x(3, 8, 128), x(3, 64), *args, buf.t, v8, k_r8, *s8, _dev(table), page,
                                     status_word=status)
        assert int(status) == 2 | (code << 8), (kind, change)
        got = buf.t.flatten(1)[:, :512].float().cpu()
        rows = {int(table[b, (int(lens[b]) - 1) // page]) * page + (int(lens[b]) - 1) % page for b in range(3) if b not in bad}
        assert set(torch.nonzero(got.any(1)).flatten().tolist()) == rows, (kind, change)
        buf.check(kind)


# ------------------------------------------------------------------ attention


def _bounds(p, scale_v, v8, x_err, rounded, terms):
    """Element-wise error bound of softmax(x) V from the kernel's roundings: weights cut to two terms by way of fp16 (2^-12),
    scores off by x_err (twice: numerator and sum), `rounded` of the result for the output's type.  Of a weight in [1, 2) the
    first term, E4M3, leaves at most 2^-4 (half of its spacing 2^-3).  The second one as E4M3 has the spacing 2^-8 there, in
    [2^-5, 2^-4): it leaves 2^-9.  As E5M2 (`terms`: the absorb path beyond 64 query rows and the tokens-on-M kernel's workers) it has 2^-7 and leaves 2^-8."""
    w = p * scale_v  # [rows, T]
    mag = np.abs(v8)
    rel = w @ mag
    floor = 2.0 ** -20 * w.max(axis=1, keepdims=True) * mag.sum(axis=0)[None]
    return rel * ({"e4m3": 2.0 ** -9, "e5m2": 2.0 ** -8}[terms] + 2.0 ** -12 + 2 * x_err + rounded) + floor


def _attend(q, x, v8, scale_v, limits):
    """q rows' softmax over their first limits[r] tokens; returns (o, lse, p) in 64 bits.  x [rows, T]."""
    o, lse = np.zeros((x.shape[0], v8.shape[1])), np.full(x.shape[0], -np.inf)
    p = np.zeros_like(x)
    for r, n in enumerate(limits):
        if n <= 0:
            continue
        m = x[r, :n].max()
        e = np.exp(x[r, :n] - m)
        p[r, :n] = e / e.sum()
        lse[r] = m + math.log(e.sum())
        o[r] = (p[r, :n] * scale_v[:n]) @ v8[:n]
    return o, lse, p


def _check_attention(path, dims, lens, s_q, page, splits, seed=11, gain=1.0, dtype=torch.bfloat16, dirty=True, hot=None,
                     scale=None):
    """One call (partials, and merged) over random pages against 64 bits.  dirty: NaN codes in every row that no sequence owns.
    hot: the token whose key is every query's, scaled to take the larger part of the weight."""
    rng = np.random.default_rng(seed)
    d = B.make_dims(**dims)
    h, g, d_h, r_kv, d_r = (dims[k] for k in ("h_q", "g", "d_h", "r_kv", "d_r"))
    heads = 1 if path == "absorb" else g
    table, n_pages = _table(rng, lens, page)
    rows = n_pages * page
    owned = np.zeros(rows, bool)
    for b, t in enumerate(lens):
        for i in range(t):
            owned[int(table[b, i // page]) * page + i % page] = True

    def plane(n_heads, width):
        codes = O.e4m3_encode(rng.standard_normal((rows, n_heads, width)).astype(np.float32) * 40)
        if dirty:
            codes[~owned] = 0x7F
        return codes, (2.0 ** rng.integers(-9, -4, size=(n_pages, n_heads))).astype(np.float32)

    width = r_kv + d_r if path == "absorb" else d_h + d_r
    dv = r_kv if path == "absorb" else d_h
    Bn = len(lens)
    q = torch.from_numpy((rng.standard_normal((Bn, s_q, h, width)) * gain * math.sqrt((d_h + d_r) / width)).astype(np.float32)).to(dtype)
    if path == "absorb":
        planes = [plane(1, width)]
    else:
        planes = [plane(g, d_h), plane(g, d_h), plane(1, d_r)]
    if hot is not None and path == "absorb":
        row = int(table[0, hot // page]) * page + hot % page
        planes[0][0][row, 0] = O.e4m3_encode(np.sign(_f64(q)[0, 0, 0]).astype(np.float32) * 100)
    scale = 1.0 / math.sqrt(d_h + d_r) if scale is None else scale
    S = abs(splits)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o_part, lse_part = Canaried((Bn, S, s_q, h, dv), torch.float32), Canaried((Bn, S, s_q, h), torch.float32)
    o_part.t.fill_(float("nan"))
    lse_part.t.fill_(float("nan"))
    out, lse = Canaried((Bn, s_q, h, dv), dtype), Canaried((Bn, s_q, h), torch.float32)
    dev = [(_dev(c), _dev(s)) for c, s in planes]
    sl = _dev(np.array(lens, np.int32))
    tail = (_dev(table), page, sl, scale, splits, o_part.t, lse_part.t, out.t, lse.t, status)
    if path == "absorb":
        B.gqla_decode_absorb_fp8_paged(d, q.cuda(), dev[0][0].view(rows, width), dev[0][1].view(-1), *tail)
    else:
        B.gqla_decode_gqa_fp8_paged(d, q.cuda(), dev[0][0], dev[1][0], dev[2][0].view(rows, d_r), dev[0][1], dev[1][1], dev[2][1].view(-1),
                                    *tail)
    torch.cuda.synchronize()
    assert int(status) == 0
    for name, c in (("o_part", o_part), ("lse_part", lse_part), ("out", out), ("lse", lse)):
        c.check(name)
    got, got_lse = _f64(out.t), _f64(lse.t)
    q64 = _f64(q)
    worst = 0.0
    pieces, sms = Bn * (S if splits > 0 else S - 1), torch.cuda.get_device_properties(0).multi_processor_count
    terms = "e5m2" if path == "absorb" and s_q * h > 64 and pieces > sms // (s_q * -(-h // 32)) else "e4m3"
    for b, T in enumerate(lens):
        at = np.array([int(table[b, t // page]) * page + t % page for t in range(T)], dtype=np.int64)
        pg = at // page
        vals = [O.e4m3_decode(c[at]) for c, _ in planes]
        for j in range(heads):
            per = h // heads
            qj = q64[b, :, j * per:(j + 1) * per].reshape(s_q * per, width)
            if path == "absorb":
                k = vals[0][:, 0] * planes[0][1][pg, 0][:, None].astype(np.float64)
                v8, sv = vals[0][:, 0, :dv], planes[0][1][pg, 0].astype(np.float64)
            else:
                k = np.concatenate([vals[0][:, j] * planes[0][1][pg, j][:, None].astype(np.float64),
                                    vals[2][:, 0] * planes[2][1][pg, 0][:, None].astype(np.float64)], axis=1)
                v8, sv = vals[1][:, j], planes[1][1][pg, j].astype(np.float64)
            x = qj @ k.T * scale
            limits = [O.visible_limit(T, s_q, p) for p in range(s_q) for _ in range(per)]
            o, l_ref, p = _attend(qj, x, v8, sv, limits)
            # scores: exact products, sums of `width` terms in fp32 (2^-24 of the largest partial sum each step at worst, taken as
            # sqrt(width) steps), and the elements of q below 2^-15 of the row's largest, off by 2^-19 of it
            x_err = 0.0
            if T:
                x_err = float(abs(scale) * (np.abs(qj) @ np.abs(k).T).max() * (2.0 ** -24 * 4 * math.sqrt(width))
                              + abs(scale) * 2.0 ** -19 * np.abs(qj).max() * np.abs(k).sum(axis=1).max() * 2.0 ** -6)
            x_err += 2.0 ** -21 * max(1.0, np.abs(x).max(initial=0.0))
            g_o = got[b, :, j * per:(j + 1) * per].reshape(s_q * per, dv)
            g_l = got_lse[b, :, j * per:(j + 1) * per].reshape(-1)
            bound = _bounds(p, sv[None], v8, x_err, torch.finfo(dtype).eps / 2, terms) if T else np.zeros_like(o)
            err = np.abs(g_o - o)
            assert np.isfinite(g_o).all(), (b, j)
            assert (err <= bound + 1e-30).all(), (b, j, float((err / np.maximum(bound, 1e-30)).max()))
            dead = np.isneginf(l_ref)
            assert np.array_equal(np.isneginf(g_l), dead)
            assert (np.abs(g_l[~dead] - l_ref[~dead]) <= x_err + 2.0 ** -22 * np.maximum(1.0, np.abs(l_ref[~dead]))).all(), (b, j)
            worst = max(worst, float((err / np.maximum(bound, 1e-30)).max(initial=0.0)))
    return worst


RAGGED = [700, 1, 385, 0, 129, 2]


@pytest.mark.parametrize("path", ["absorb", "gqa"])
@pytest.mark.parametrize("page", [16, 32, 48, 64, 128, 320])
@pytest.mark.parametrize("splits", [1, 3, -4])
def test_attention_over_pages(path, page, splits):
    _check_attention(path, CANON, RAGGED, 2, page, splits)


@pytest.mark.parametrize("page", [16, 32, 48, 64, 128, 320])
@pytest.mark.parametrize("splits", [9, -13])
def test_pairs_over_pages(page, splits):
    """More pieces than the tokens-on-M kernel has workers for these rows."""
    _check_attention("absorb", CANON, RAGGED, 2, page, splits)


@pytest.mark.parametrize("dims", [LLAMA, dict(h_q=64, g=8, d_h=128, r_kv=512, d_r=64), dict(h_q=28, g=4, d_h=128, r_kv=512, d_r=64),
                                  dict(h_q=40, g=1, d_h=128, r_kv=512, d_r=64)])
def test_pairs_head_layouts(dims):
    _check_attention("absorb", dims, [300, 5, 1, 257], 3, 64, -20)
    _check_attention("absorb", dims, [300, 5, 1, 257], 3, 64, 19)


@pytest.mark.parametrize("path", ["absorb", "gqa"])
@pytest.mark.parametrize("dims", [LLAMA, dict(h_q=64, g=8, d_h=128, r_kv=512, d_r=64), dict(h_q=28, g=4, d_h=128, r_kv=512, d_r=64),
                                  dict(h_q=20, g=20, d_h=128, r_kv=512, d_r=64), dict(h_q=40, g=1, d_h=128, r_kv=512, d_r=64),
                                  dict(h_q=1, g=1, d_h=128, r_kv=512, d_r=64)])
@pytest.mark.parametrize("s_q", [1, 3])
def test_attention_head_layouts(path, dims, s_q):
    _check_attention(path, dims, [300, 5, 1, 257], s_q, 64, -3)


@pytest.mark.parametrize("path", ["absorb", "gqa"])
@pytest.mark.parametrize("s_q", [5, 8, 40])
def test_attention_of_many_query_positions(path, s_q):
    _check_attention(path, LLAMA, [200, 41, 7], s_q, 32, -3)


@pytest.mark.parametrize("path", ["absorb", "gqa"])
@pytest.mark.parametrize("dims,page,dtype,policy", [(TINY, 7, torch.float32, "auto"), (TINY, 16, torch.bfloat16, "auto"),
                                                    (LLAMA, 64, torch.float32, "auto"), (LLAMA, 24, torch.bfloat16, "auto"),
                                                    (LLAMA, 64, torch.bfloat16, "generic")])
def test_attention_on_the_generic_kernel(path, dims, page, dtype, policy):
    B.set_policy(B.POLICY_GENERIC if policy == "generic" else B.POLICY_AUTO)
    try:
        _check_attention(path, dims, [90, 0, 1, 33], 2, page, 2, dtype=dtype)
        _check_attention(path, dims, [90, 0, 1, 33], 2, page, -3, dtype=dtype)
    finally:
        B.set_policy(B.POLICY_AUTO)


@pytest.mark.parametrize("path", ["absorb", "gqa"])
@pytest.mark.parametrize("gain", [0.02, 8.0, 40.0])
def test_attention_flat_and_peaked_scores(path, gain):
    """Scores all alike, and scores that outgrow a piece's first references many times over."""
    _check_attention(path, LLAMA, [1500, 130], 1, 64, -2, gain=gain)


@pytest.mark.parametrize("hot", [3, 700, 1999])
def test_one_key_with_most_of_the_weight(hot):
    _check_attention("absorb", LLAMA, [2000], 1, 64, -2, hot=hot)
    _check_attention("absorb", LLAMA, [2000], 1, 16, 1, hot=hot)


@pytest.mark.parametrize("gain", [0.02, 8.0, 40.0])
@pytest.mark.parametrize("s_q,page", [(1, 64), (2, 16)])
def test_pairs_flat_and_peaked_scores(gain, s_q, page):
    _check_attention("absorb", CANON, [1500, 130, 3], s_q, page, -2, gain=gain)
    _check_attention("absorb", CANON, [1500, 130, 3], s_q, page, -14, gain=gain)


@pytest.mark.parametrize("hot", [3, 1999])
def test_pairs_one_key_with_most_of_the_weight(hot):
    _check_attention("absorb", CANON, [2000, 1], 1, 64, -40, hot=hot)
    _check_attention("absorb", CANON, [2000] + [700] * 39, 1, 64, 1, hot=hot)


@pytest.mark.parametrize("path,dims", [("absorb", CANON), ("absorb", LLAMA), ("gqa", LLAMA)])
@pytest.mark.parametrize("scale", [-0.05, 0.0])
def test_attention_scale_of_any_sign(path, dims, scale):
    _check_attention(path, dims, [300, 1, 150], 2, 32, -3, scale=scale)
    if dims is CANON:
        _check_attention(path, dims, [300, 1, 150], 2, 32, -14, scale=scale)


@pytest.mark.parametrize("path,dims", [("absorb", CANON), ("absorb", LLAMA), ("gqa", LLAMA), ("gqa", CANON)])
@pytest.mark.parametrize("splits", [1, -3, -20, 20])
def test_attention_over_nothing(path, dims, splits):
    """Sequences without a token, and of fewer tokens than query positions."""
    _check_attention(path, dims, [0, 0, 0], 2, 64, splits)
    _check_attention(path, dims, [1, 0, 2], 4, 16, splits)


@pytest.mark.parametrize("path,dims,batch", [("absorb", CANON, 60), ("absorb", LLAMA, 110), ("gqa", LLAMA, 14)])
@pytest.mark.parametrize("splits", [-2, -5])
def test_a_piece_per_sequence(rng, path, dims, batch, splits):
    """About a sequence per worker: each goes to one worker whole, and the slots behind its first are empty."""
    workers = B.gqla_fp8_paged_workers(B.make_dims(**dims), torch.bfloat16, 1, 64, path)
    assert workers // 2 < batch <= workers
    lens = [int(t) for t in rng.integers(300, 640, size=batch)]
    lens[3], lens[batch // 2], lens[-1] = 0, 1, 0
    _check_attention(path, dims, lens, 1, 64, splits)


def test_one_long_sequence_on_every_pair(rng):
    _check_attention("absorb", CANON, [9000], 1, 64, -72)


def test_large_batch_plan(rng):
    """More sequences than one warp plans for."""
    lens = [int(t) for t in rng.integers(0, 200, size=150)]
    _check_attention("gqa", LLAMA, lens, 1, 16, -3)


def test_page_numbers_past_32_bits_of_bytes():
    """A pool of more than 2^32 bytes: the last pages are reached."""
    d, page, n_pages = B.make_dims(**LLAMA), 64, 120_000
    cache = torch.zeros((n_pages * page, 576), dtype=torch.uint8, device="cuda")
    scale = torch.ones(n_pages, device="cuda")
    lens = torch.tensor([100], dtype=torch.int32, device="cuda")
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    c = torch.randn((100, 512), generator=g, device="cuda").bfloat16()
    k_r = torch.randn((100, 64), generator=g, device="cuda").bfloat16()
    B.gqla_append_rope_fp8(d, c, k_r, torch.tensor([0, 100], dtype=torch.int32, device="cuda"), lens, _dev(_angles(100, 64)), "pairs",
                           cache, scale, table, page)
    q = torch.randn((1, 1, 32, 576), generator=g, device="cuda").bfloat16()
    o_part, lse_part = torch.empty((1, 2, 1, 32, 512), device="cuda"), torch.empty((1, 2, 1, 32), device="cuda")
    out = torch.empty((1, 1, 32, 512), dtype=torch.bfloat16, device="cuda")
    B.gqla_decode_absorb_fp8_paged(d, q, cache, scale, table, page, lens, 0.07, -2, o_part, lse_part, out)
    at = torch.cat([torch.arange(64) + (n_pages - 1) * page, torch.arange(36) + (n_pages - 2) * page]).cuda()
    k = (cache[at].view(torch.float8_e4m3fn).double() * scale[at // page].double()[:, None])
    assert float((k[:, :512] - c.double()).abs().max()) <= 2.0 ** -4 * float(c.abs().max())
    assert not cache[:1000 * page].any()
    p = torch.softmax(q[0, 0].double() @ k.T * 0.07, -1)
    assert float((out[0, 0].double() - p @ k[:, :512]).abs().max()) <= 2.0 ** -7 * float((p @ k[:, :512].abs()).max())


# ------------------------------------------------------------------ a server's run


def _weights(dims, seed=2):
    g = torch.Generator().manual_seed(seed)
    shape = (dims["g"], dims["r_kv"], dims["d_h"])
    return [(torch.randn(shape, generator=g) / math.sqrt(dims["r_kv"])).bfloat16().cuda() for _ in range(2)]


@pytest.mark.parametrize("dims,style", [(CANON, "pairs"), (LLAMA, "halves")])
def test_prompt_then_steps_on_both_paths(dims, style):
    """Prompts, then steps of one and two tokens, the same on the bf16 cache, the E4M3 latent pages and the E4M3 planes: each step's
    outputs against 64 bits on the caches as they were before rounding, within E4M3's rounding; bf16 within its own."""
    g = torch.Generator().manual_seed(4)
    page, lens, steps = 32, [70, 1, 200], [1, 2, 1]
    total = [t + sum(steps) for t in lens]
    rng = np.random.default_rng(3)
    table_np, n_pages = _table(rng, total, page)
    table, rope = _dev(np.maximum(table_np, 0)), _dev(_angles(max(total), dims["d_r"]))
    w_uk, w_uv = _weights(dims)
    h, gr, d_h, r_kv, d_r = (dims[k] for k in ("h_q", "g", "d_h", "r_kv", "d_r"))
    scale = 1.0 / math.sqrt(d_h + d_r)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pool = torch.zeros((n_pages * page, r_kv + d_r), dtype=torch.bfloat16, device="cuda")
    plain = GqlaDecoder(**dims, w_uk=w_uk, w_uv=w_uv, cache=pool, seq_start=None, seqlens=sl, scale=scale, block_table=table, page_size=page)
    latent, planes = (GqlaFp8PagedDecoder(**dims, w_uk=w_uk, w_uv=w_uv, n_pages=n_pages, page_size=page, block_table=table, seqlens=sl,
                                          scale=scale, rope=rope, style=style, expanded=e) for e in (False, True))
    rows = [[] for _ in lens]
    od = O.Dims(h, gr, d_h, r_kv, d_r)
    for step, s_q in enumerate([0] + steps):
        new = [s_q or t for t in lens]
        if s_q:
            sl += s_q
        n = sum(new)
        starts = _dev(_starts(new))
        c = torch.randn((n, r_kv), generator=g).bfloat16().cuda()
        k_r = torch.randn((n, d_r), generator=g).bfloat16().cuda()
        q = torch.randn((n, h, d_h + d_r), generator=g).bfloat16().cuda()
        pos = [t for _, t in O.new_row_places(_starts(new), sl.tolist())]
        turned = O.rope_turn(_f64(k_r), pos, _f64(rope), style)
        for i, (b, _) in enumerate(O.new_row_places(_starts(new), sl.tolist())):
            rows[b].append(np.concatenate([_f64(c)[i], turned[i]]))
        q_gqa = q.clone()
        q_bf = plain.append(c, k_r, starts, rope, style, q[..., d_h:])
        q_lat = latent.append(c, k_r, starts, q[..., d_h:])
        planes.append_expanded(c, k_r, starts, q_gqa)
        assert torch.equal(q_bf, q_lat) and torch.equal(q_bf, q_gqa[..., d_h:]) and torch.equal(q_gqa[..., :d_h], q[..., :d_h])
        if not s_q:
            continue
        view = lambda t: t.view(len(lens), s_q, h, -1).contiguous()  # noqa: E731
        q_c, q_r = view(q[..., :d_h]), view(q_bf)
        got = {"bf16": plain.absorb_step(q_c, q_r, -3), "latent": latent.absorb_step(q_c, q_r, -3),
               "latent_apart": latent.absorb_step(q_c, q_r, 2, fused_tail=False).clone(), "planes": planes.gqa_step(view(q_gqa), -3)}
        latent.absorb_step(q_c, q_r, -3)
        flat = np.concatenate([np.array(r) for r in rows])
        start = np.concatenate([[0], np.cumsum([len(r) for r in rows])])[:-1]
        ref = O.absorb_path(od, _f64(q_c), _f64(q_r), _f64(w_uk), _f64(w_uv), flat, start, np.array(sl.tolist()), s_q, scale)
        for name, o in got.items():
            err = np.linalg.norm(_f64(o) - ref) / np.linalg.norm(ref)
            # E4M3 rows are off by 2^-4 / sqrt(3) of each element at most in the mean square, keys and values both; bf16: 2^-8 in a few places
            assert err <= (2.0 ** -6 if name == "bf16" else 2 * 2.0 ** -4), (step, name, err)
    for dec in (plain, latent, planes):
        dec.check_status()


def test_steps_captured_and_replayed(rng):
    """A step captured into a graph with its append: replays with other rows in the same tensors give what eager calls give;
    two graphs of one decoder are replayed in turn."""
    dims, page, n_pages = LLAMA, 16, 40
    w_uk, w_uv = _weights(dims)
    table = _dev(rng.permutation(n_pages).reshape(4, 10).astype(np.int32))
    rope = _dev(_angles(160, 64))

    def make():
        sl = torch.tensor([20, 31, 100, 1], dtype=torch.int32, device="cuda")
        dec = GqlaFp8PagedDecoder(**dims, w_uk=w_uk, w_uv=w_uv, n_pages=n_pages, page_size=page, block_table=table, seqlens=sl, scale=0.07,
                                  rope=rope)
        g = torch.Generator(device="cuda").manual_seed(8)
        lens = sl.tolist()
        c = torch.randn((sum(lens), 512), generator=g, device="cuda").bfloat16()
        k_r = torch.randn((sum(lens), 64), generator=g, device="cuda").bfloat16()
        dec.append(c, k_r, _dev(_starts(lens)))
        return dec, sl

    starts = _dev(_starts([1] * 4))
    c, k_r, q_c, q_r = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((4, 512), (4, 64), (4, 1, 32, 128), (4, 32, 64)))

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (c, k_r, q_c, q_r):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    def step(dec):
        return dec.absorb_step(q_c, dec.append(c, k_r, starts, q_r).view(4, 1, 32, 64), -2)

    eager, sl_e = make()
    want = []
    for seed in range(4):
        fill(seed)
        sl_e += 1
        want.append(step(eager).clone())
    dec, sl = make()
    sl += 1
    fill(0)
    (run1, out1), (run2, out2) = dec.capture(step, dec), dec.capture(step, dec)
    for seed in range(4):
        fill(seed)
        if seed:
            sl += 1
        (run1, run2)[seed % 2]()
        assert torch.equal((out1, out2)[seed % 2], want[seed]), seed
    assert torch.equal(dec.cache, eager.cache) and torch.equal(dec.page_scale, eager.page_scale)


def test_calls_on_another_stream():
    """Calls follow the current stream, and two of them at once on two streams do not disturb each other."""
    dims, page = LLAMA, 64
    d = B.make_dims(**dims)
    g = torch.Generator(device="cuda").manual_seed(3)
    table = torch.arange(64, dtype=torch.int32, device="cuda").view(4, 16)
    sl = torch.tensor([1000, 900, 800, 1], dtype=torch.int32, device="cuda")
    codes = torch.randint(0, 0x7E, (64 * page, 576), generator=g, device="cuda", dtype=torch.uint8)
    scale = torch.full((64,), 2.0 ** -9, device="cuda")
    q = [torch.randn((4, 1, 32, 576), generator=g, device="cuda").bfloat16() for _ in range(2)]

    def call(x, bufs):
        B.gqla_decode_absorb_fp8_paged(d, x, codes, scale, table, page, sl, 0.05, -8, *bufs)

    def buffers():
        return (torch.empty((4, 8, 1, 32, 512), device="cuda"), torch.empty((4, 8, 1, 32), device="cuda"),
                torch.empty((4, 1, 32, 512), dtype=torch.bfloat16, device="cuda"))

    want = []
    for x in q:
        b = buffers()
        call(x, b)
        want.append(b[2])
    streams = [torch.cuda.Stream() for _ in q]
    got = [buffers() for _ in q]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, b, s in zip(q, got, streams):
            with torch.cuda.stream(s):
                call(x, b)
    torch.cuda.synchronize()
    for b, w in zip(got, want):
        assert torch.equal(b[2], w)


def test_refusals_of_the_binding():
    d, page = B.make_dims(**LLAMA), 16
    x = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    good = dict(c=x(2, 512), k_r=x(2, 64), new_start=i32(3), seqlens=i32(2), rope=x(8, 64, t=torch.float32), style="pairs",
                cache8=x(64, 576, t=torch.uint8), page_scale=x(4, t=torch.float32), block_table=i32(2, 2), page_size=page)
    B.gqla_append_rope_fp8(d, **good)
    bad = [dict(style="half"), dict(c=x(2, 511)), dict(c=x(2, 512, t=torch.float32)), dict(k_r=x(3, 64)), dict(new_start=i32(2)),
           dict(seqlens=i32(3)), dict(rope=x(8, 32, t=torch.float32)), dict(rope=x(8, 64)), dict(cache8=x(63, 576, t=torch.uint8)),
           dict(cache8=x(64, 576)), dict(page_scale=x(5, t=torch.float32)), dict(block_table=i32(3, 2)), dict(page_size=0),
           dict(q_r=x(2, 32, 64)), dict(q_r=x(2, 32, 64), q_out=x(2, 31, 64)), dict(c=x(2, 1024)[:, ::2]), dict(c=x(2, 512).cpu()),
           dict(c=x(2, 512, t=torch.float16), k_r=x(2, 64, t=torch.float16))]
    for change in bad:
        with pytest.raises(B.GqlaError):
            B.gqla_append_rope_fp8(d, **{**good, **change})
    dec = dict(q_hat=x(2, 1, 32, 576), cache8=good["cache8"], page_scale=good["page_scale"], block_table=good["block_table"], page_size=page,
               seqlens=good["seqlens"], scale=0.1, num_splits=2, o_part=x(2, 2, 1, 32, 512, t=torch.float32),
               lse_part=x(2, 2, 1, 32, t=torch.float32))
    B.gqla_decode_absorb_fp8_paged(d, **dec)
    for change in (dict(q_hat=x(2, 1, 32, 575)), dict(q_hat=x(2, 1, 32, 576, t=torch.float16)), dict(num_splits=3), dict(num_splits=0),
                   dict(o_part=x(2, 2, 1, 32, 512)), dict(out=x(2, 1, 32, 128)), dict(out=x(2, 1, 32, 512, t=torch.float32)),
                   dict(lse=x(2, 1, 32, t=torch.float32)), dict(seqlens=i32(2).cpu()), dict(page_scale=x(4)), dict(block_table=i32(2, 2).long())):
        with pytest.raises(B.GqlaError):
            B.gqla_decode_absorb_fp8_paged(d, **{**dec, **change})
