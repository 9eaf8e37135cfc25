"""Appends of the sizes that prompts and serving batches have: several rows a warp, searches of more than one round over the sequences,
runs of sequences without new rows.  Cache rows and queries against complex multiplication in 64 bits, E4M3 pages bit for bit against the
oracle."""
import numpy as np
import pytest
import torch

from oracle import gqla_oracle as O
from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild
from tests.parity_util import Canaried
from tests.test_gpu_fp8_paged import _angles, _dev, _exact_turns, _f64, _few_bits, _pages, _same_codes, _starts, _table

pytestmark = pytest.mark.gpu

CANON = dict(h_q=2, g=1, d_h=128, r_kv=512, d_r=64)
TINY = dict(h_q=6, g=2, d_h=10, r_kv=20, d_r=6)
SMALL = dict(h_q=2, g=2, d_h=16, r_kv=32, d_r=16)  # vectors of eight


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gbuild.build()
    assert torch.cuda.is_available()
    B.lib()


def _batch(kind, batch, seed=7):
    """Lengths and new rows."""
    rng = np.random.default_rng(seed + batch)
    if kind == "prompts":  # 8192 rows and more, no multiple of four, of sequences some of which miss their first rows
        new = rng.multinomial(8192 + 4 * batch + 3, np.ones(batch) / batch)
        lens = np.maximum(new + rng.integers(-2, 3, size=batch) * (rng.random(batch) < 0.4), 0)
    elif kind == "steps":
        lens, new = rng.integers(1, 60, size=batch), np.ones(batch, dtype=np.int64)
    elif kind == "few":  # long runs of sequences without a new row, at the ends too
        lens, new = rng.integers(0, 60, size=batch), np.zeros(batch, dtype=np.int64)
        for i in rng.choice(np.arange(1, batch - 1), size=max(2, batch // 20), replace=False):
            new[i] = rng.integers(1, 4)
            lens[i] += new[i]
    else:  # "short prompts": more rows than pages and two units a sequence
        new = rng.integers(0, 40, size=batch) * (rng.random(batch) < 0.6)
        lens = new + rng.integers(0, 30, size=batch)
        lens[batch // 2] = new[batch // 2] = 200
    return [int(t) for t in lens], [int(k) for k in new]


def _turned(x, pos, table, style):
    half = x.shape[-1] // 2
    w = (table[pos, :half] + 1j * table[pos, half:].astype(np.float64)).reshape(len(pos), *([1] * (x.ndim - 2)), half)
    a, b = (x[..., 0::2], x[..., 1::2]) if style == "pairs" else (x[..., :half], x[..., half:])
    z, out = (a + 1j * b) * w, np.empty_like(x)
    if style == "pairs":
        out[..., 0::2], out[..., 1::2] = z.real, z.imag
    else:
        out[..., :half], out[..., half:] = z.real, z.imag
    return out


@pytest.mark.parametrize("dims,dtype,paged,style", [(CANON, torch.bfloat16, True, "pairs"), (CANON, torch.float32, False, "halves"),
                                                    (TINY, torch.bfloat16, False, "halves"), (TINY, torch.float32, True, "pairs"),
                                                    (SMALL, torch.bfloat16, True, "halves")])
@pytest.mark.parametrize("kind,batch", [("prompts", 1), ("prompts", 5), ("prompts", 33), ("prompts", 1025), ("steps", 33), ("steps", 64),
                                        ("steps", 1025), ("few", 40), ("few", 1500)])
def test_append_rope_of_many_rows_and_sequences(dims, dtype, paged, style, kind, batch):
    lens, new = _batch(kind, batch)
    rng = np.random.default_rng(1)
    d, n, page = B.make_dims(**dims), sum(new), 24
    assert kind != "prompts" or n >= 8192 and n % 4 == 3
    table, n_pages = _table(rng, lens, page)
    starts = np.cumsum([0] + [t + 1 for t in lens])[:-1].astype(np.int64)
    rows = n_pages * page if paged else int(sum(lens)) + batch
    c, k_r, q = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dtype)
                 for s in ((n, dims["r_kv"]), (n, dims["d_r"]), (n, dims["h_q"], dims["d_r"])))
    rope = _angles(max(lens) + 1, dims["d_r"])
    cache, q_out = Canaried((rows, dims["r_kv"] + dims["d_r"]), dtype), Canaried(q.shape, dtype)
    cache.t.fill_(3.0)
    q_out.t.fill_(9.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.gqla_append_rope(d, c.cuda(), k_r.cuda(), _dev(_starts(new)), _dev(np.array(lens, np.int32)), _dev(rope), style, cache.t,
                       None if paged else _dev(starts), _dev(table) if paged else None, page if paged else 0, q.cuda(), q_out.t, status)
    seq, pos = (np.array(x) for x in zip(*O.new_row_places(_starts(new), lens)))
    kept = pos >= 0
    seq, pos = seq[kept], pos[kept]
    at = table[seq, pos // page].astype(np.int64) * page + pos % page if paged else starts[seq] + pos
    got = _f64(cache.t)
    want = np.full_like(got, 3.0)
    want[at, :dims["r_kv"]] = _f64(c)[kept]
    want[at, dims["r_kv"]:] = got[at, dims["r_kv"]:]
    assert np.array_equal(got, want)
    # two fp32 products and a sum, then one rounding to the storage type, of the pair's size
    eps = torch.finfo(dtype).eps / 2 + 3 * 2.0 ** -24
    for g, x in ((got[at, dims["r_kv"]:], _f64(k_r)[kept]), (_f64(q_out.t)[kept], _f64(q)[kept])):
        assert np.abs(g - _turned(x, pos, rope, style)).max(initial=0.0) <= eps * np.abs(x).max(initial=0.0) * 2 ** 0.5
    assert (_f64(q_out.t)[~kept] == 9.0).all()
    cache.check("cache")
    q_out.check("q_out")
    assert int(status) == 0


@pytest.mark.parametrize("dims,dtype", [(TINY, torch.float32), (SMALL, torch.bfloat16)])
@pytest.mark.parametrize("kind,batch,page", [("steps", 33, 16), ("steps", 64, 8), ("steps", 1025, 16), ("few", 40, 16), ("few", 1500, 8),
                                             ("short prompts", 33, 16), ("short prompts", 64, 24), ("short prompts", 1025, 16)])
def test_append_fp8_of_many_sequences_bit_for_bit(dims, dtype, kind, batch, page):
    lens, new = _batch(kind, batch)
    rng = np.random.default_rng(2)
    d, n = B.make_dims(**dims), sum(new)
    by_pages = n // (1 << (page.bit_length() - 1)) + 2 * batch
    assert (n >= by_pages) == (kind == "short prompts")
    table, n_pages = _table(rng, lens, page)
    rope = _exact_turns(rng, max(lens) + 1, dims["d_r"])
    step = (_dev(_starts(new)), _dev(np.array(lens, np.int32)), _dev(rope), "pairs")
    pos = [max(t, 0) for _, t in O.new_row_places(_starts(new), lens)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    g, d_h, d_r, r_kv = (dims[k] for k in ("g", "d_h", "d_r", "r_kv"))
    c, k_c, v, k_r = (_few_bits(rng, (n, *s), dtype) for s in ((r_kv,), (g, d_h), (g, d_h), (d_r,)))
    turned = _turned(_f64(k_r), pos, rope, "pairs")
    q = _few_bits(rng, (n, dims["h_q"], d_r), dtype)

    def buffers(heads, width, shape, scale_shape):
        codes, scale = _pages(rng, n_pages, page, heads, width)
        a, b = Canaried((n_pages * page, *shape), torch.uint8), Canaried((n_pages, *scale_shape), torch.float32)
        a.t.copy_(torch.from_numpy(codes.reshape(a.t.shape)))
        b.t.copy_(torch.from_numpy(scale.reshape(b.t.shape)))
        return a, b, codes, scale

    latent = buffers(1, r_kv + d_r, (r_kv + d_r,), ())
    planes = [buffers(g, d_h, (g, d_h), (g,)), buffers(g, d_h, (g, d_h), (g,)), buffers(1, d_r, (d_r,), ())]
    q_out = [Canaried(q.shape, dtype) for _ in range(2)]
    B.gqla_append_rope_fp8(d, c.cuda(), k_r.cuda(), *step, latent[0].t, latent[1].t, _dev(table), page, q.cuda(), q_out[0].t, status)
    B.gqla_append_planes_fp8(d, k_c.cuda(), v.cuda(), k_r.cuda(), *step, *(p[0].t for p in planes), *(p[1].t for p in planes), _dev(table),
                             page, q.cuda(), q_out[1].t, status)
    assert int(status) == 0
    for (a, b, codes, scale), rows in zip([latent, *planes], [np.concatenate([_f64(c), turned], axis=1)[:, None], _f64(k_c), _f64(v),
                                                              turned[:, None]]):
        want_codes, want_scale = O.append_pages_e4m3(rows, codes, scale, _starts(new), lens, table, page)
        assert np.array_equal(b.t.cpu().numpy().reshape(scale.shape), want_scale)
        assert _same_codes(a.t.cpu().numpy().reshape(codes.shape), want_codes).all()
        a.check("codes")
        b.check("scales")
    want = torch.from_numpy(_turned(_f64(q), pos, rope, "pairs")).to(dtype)  # (exact in fp32, then rounded once)
    for o in q_out:
        assert torch.equal(o.t.cpu(), want)
        o.check("q_out")
