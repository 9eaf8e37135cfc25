"""Host side of the append calls and of attention over E4M3 pages (no GPU): argument errors return before anything is launched,
the oracle's statements of the rotation, the scales and the pages against hand-worked and library values, the warps' votes."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import gqla_oracle as O
from paper_2605_15250_b200 import binding as B
from paper_2605_15250_b200 import build as gbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    gbuild.build()


P = ctypes.c_void_p(0x1000)  # aligned, never dereferenced on these paths
ODD = ctypes.c_void_p(0x1004)
OK, NULL, SHAPE, ALIGN, DTYPE = 0, 1, 2, 3, 4


def _d(**change):
    return ctypes.byref(B.make_dims(**{**dict(h_q=128, g=8, d_h=128, r_kv=512, d_r=64), **change}))


APPEND = dict(dims=None, dtype=0, B=2, n=5, new_start=P, seqlens=P, c=P, c_stride=512, k_r=P, k_r_stride=64, rope=P, rope_rows=100,
              style=0, q_r=P, q_row=8192, q_head=64, q_out=P, o_row=8192, o_head=64)


@pytest.mark.parametrize("change,code", [
    (dict(dims=_d(h_q=127)), SHAPE), (dict(dims=0), NULL), (dict(dtype=2), DTYPE), (dict(B=-1), SHAPE), (dict(n=-1), SHAPE),
    (dict(n=1 << 31), SHAPE), (dict(style=2), SHAPE), (dict(dims=_d(d_r=63)), SHAPE), (dict(new_start=None), NULL),
    (dict(seqlens=None), NULL), (dict(c=None), NULL), (dict(k_r=None), NULL), (dict(rope=None), NULL), (dict(rope_rows=-1), SHAPE),
    (dict(c_stride=511), SHAPE), (dict(k_r_stride=63), SHAPE), (dict(q_r=None), NULL), (dict(q_out=None), NULL),
    (dict(q_head=63), SHAPE), (dict(o_row=63), SHAPE), (dict(n=0), OK), (dict(B=0), OK)])
@pytest.mark.parametrize("call", ["rope", "fp8", "planes"])
def test_append_argument_errors(call, change, code):
    a = {**APPEND, "dims": _d(), **change}
    dims = None if a["dims"] == 0 else a["dims"]
    front = [dims, a["dtype"], a["B"], a["n"], a["new_start"], a["seqlens"]]
    mid = [a[k] for k in ("k_r", "k_r_stride", "rope", "rope_rows", "style", "q_r", "q_row", "q_head", "q_out", "o_row", "o_head")]
    L = B.lib()
    if call == "rope":
        got = L.gqla_append_rope(*front, a["c"], a["c_stride"], *mid, P, 576, 640, None, P, 4, 64, None, None)
    elif call == "fp8":
        got = L.gqla_append_rope_fp8(*front, a["c"], a["c_stride"], *mid, P, 576, 640, P, P, 4, 64, None, None)
    else:
        if "c_stride" in change:
            return
        got = L.gqla_append_planes_fp8(*front, a["c"], P, *mid, P, P, P, 64, 640, P, P, P, P, 4, 64, None, None)
    assert got == code


def test_append_errors_of_the_caches():
    L = B.lib()
    front = [_d(), 0, 2, 5, P, P, P, 512]
    mid = [P, 64, P, 100, 0, None, 0, 0, None, 0, 0]
    rope = lambda *a: L.gqla_append_rope(*front, *mid, *a, None, None)  # noqa: E731
    assert rope(None, 576, 640, None, P, 4, 64) == NULL and rope(P, 575, 640, None, P, 4, 64) == SHAPE
    assert rope(P, 576, -1, None, P, 4, 64) == SHAPE and rope(P, 576, 640, P, P, 4, 64) == NULL
    assert rope(P, 576, 640, None, None, 4, 64) == NULL
    assert rope(P, 576, 640, None, P, 0, 64) == SHAPE and rope(P, 576, 640, None, P, 4, 0) == SHAPE
    fp8 = lambda *a: L.gqla_append_rope_fp8(*front, *mid, *a, None, None)  # noqa: E731
    assert fp8(None, 576, 640, P, P, 4, 64) == NULL and fp8(P, 576, 640, None, P, 4, 64) == NULL
    assert fp8(P, 576, 640, P, None, 4, 64) == NULL and fp8(P, 575, 640, P, P, 4, 64) == SHAPE
    assert fp8(P, 576, 1 << 31, P, P, 4, 64) == SHAPE and fp8(P, 576, 640, P, P, 4, 0) == SHAPE
    front[6:] = [P, P]
    planes = lambda *a: L.gqla_append_planes_fp8(*front, *mid, *a, None, None)  # noqa: E731
    good = [P, P, P, 64, 640, P, P, P, P, 4, 64]
    for i in (0, 1, 2, 5, 6, 7, 8):
        assert planes(*good[:i], None, *good[i + 1:]) == NULL
    assert planes(*good[:3], 63, *good[4:]) == SHAPE and planes(*good[:4], -1, *good[5:]) == SHAPE
    assert planes(*good[:9], 0, 64) == SHAPE and planes(*good[:10], 0) == SHAPE


@pytest.mark.parametrize("change,code", [
    (dict(dims=_d(h_q=127)), SHAPE), (dict(dims=0), NULL), (dict(dtype=2), DTYPE), (dict(B=-1), SHAPE), (dict(s_q=0), SHAPE),
    (dict(splits=0), SHAPE), (dict(splits=-1), SHAPE), (dict(page_size=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(rows=-1), SHAPE),
    (dict(rows=1 << 31), SHAPE), (dict(q=None), NULL), (dict(k=None), NULL), (dict(k_scale=None), NULL), (dict(table=None), NULL),
    (dict(seqlens=None), NULL), (dict(o_part=None), NULL), (dict(lse_part=None), NULL), (dict(out=None), NULL), (dict(q=ODD), ALIGN),
    (dict(k=ODD), ALIGN), (dict(o_part=ODD), ALIGN), (dict(out=ODD), ALIGN), (dict(B=0), OK)])
@pytest.mark.parametrize("path", ["absorb", "gqa"])
def test_decode_argument_errors(path, change, code):
    a = {**dict(dims=_d(), dtype=0, B=2, s_q=1, splits=2, rows=640, page_size=64, max_pages=4, q=P, k=P, k_scale=P, table=P, seqlens=P,
                o_part=P, lse_part=P, out=P), **change}
    dims = None if a["dims"] == 0 else a["dims"]
    front = [dims, a["dtype"], a["B"], a["s_q"], 0.1, a["splits"], a["q"], a["k"]]
    tail = [a["table"], a["max_pages"], a["page_size"], a["seqlens"], a["o_part"], a["lse_part"], a["out"], P, None, None]
    if path == "absorb":
        got = B.lib().gqla_decode_absorb_fp8_paged(*front, 576, a["rows"], a["k_scale"], *tail)
    else:
        got = B.lib().gqla_decode_gqa_fp8_paged(*front, P, P, 64, a["rows"], a["k_scale"], P, P, *tail)
    assert got == code


def test_decode_errors_of_one_path():
    L = B.lib()
    front, tail = [_d(), 0, 2, 1, 0.1, 2, P, P], [P, 4, 64, P, P, P, None, None, None, None]
    assert L.gqla_decode_absorb_fp8_paged(*front, 575, 640, P, *tail) == SHAPE
    gqa = L.gqla_decode_gqa_fp8_paged
    assert gqa(*front, None, P, 64, 640, P, P, P, *tail) == NULL and gqa(*front, P, None, 64, 640, P, P, P, *tail) == NULL
    assert gqa(*front, P, P, 63, 640, P, P, P, *tail) == SHAPE and gqa(*front, P, P, 64, 640, P, None, P, *tail) == NULL
    assert gqa(*front, P, P, 64, 640, P, P, None, *tail) == NULL and gqa(*front, ODD, P, 64, 640, P, P, P, *tail) == ALIGN
    wide = _d(r_kv=1024)
    assert L.gqla_decode_absorb_fp8_paged(wide, 0, 2, 1, 0.1, 2, P, P, 1088, 640, P, *tail) == 5  # values over 512 wide: no kernel
    d = B.make_dims(128, 8, 128, 512, 64)
    assert B.gqla_fp8_paged_workers(d, torch.float32, 1, 64, "absorb") == 0 and B.gqla_fp8_paged_workers(d, torch.bfloat16, 1, 24, "gqa") == 0
    assert B.gqla_fp8_paged_workers(d, torch.bfloat16, 0, 64, "gqa") == -1


def test_warps_of_the_paged_kernels_leave_by_vote():
    """Block barriers have no limit, so the warps that meet in them leave a loop together, by a vote on their failed waits."""
    for name in ("tc_decode_fp8_paged.cuh", "tc_decode_fp8_pair.cuh"):
        path = os.path.join(ROOT, "paper_2605_15250_b200", "csrc", name)
        text = re.sub(r"//[^\n]*", "", open(path).read())
        kernel = text.split("__global__")[1]
        softmax = kernel.split("vote_any(")[0].rfind("} else")
        assert ".raised()" not in kernel[softmax:], name
        assert re.search(r"if \(vote_any\(\w+, !okl, [^;{]*\)\) \{ ok = false; break; \}", kernel), name


# ------------------------------------------------------------------ the oracle's statements


def test_oracle_rotation_by_hand():
    """Quarter and half turns by hand; a turn by any angle against complex multiplication; position 0 leaves a row alone."""
    table = np.array([[1.0, 1.0, 0.0, 0.0], [0.0, -1.0, 1.0, 0.0]])
    x = np.array([[1.0, 2.0, 3.0, 4.0], [1.0, 2.0, 3.0, 4.0]])
    assert np.array_equal(O.rope_turn(x, [0, 1], table, "pairs"), [[1, 2, 3, 4], [-2, 1, -3, -4]])
    assert np.array_equal(O.rope_turn(x, [0, 1], table, "halves"), [[1, 2, 3, 4], [-3, -2, 1, -4]])
    rng = np.random.default_rng(0)
    ang = rng.uniform(0, 6.28, size=(5, 3))
    table, x = np.concatenate([np.cos(ang), np.sin(ang)], axis=1), rng.standard_normal((5, 2, 6))
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * ang)[:, None]
    got = O.rope_turn(x, range(5), table, "pairs")
    assert np.allclose(got[..., 0::2], z.real, atol=1e-14) and np.allclose(got[..., 1::2], z.imag, atol=1e-14)
    z = (x[..., :3] + 1j * x[..., 3:]) * np.exp(1j * ang)[:, None]
    got = O.rope_turn(x, range(5), table, "halves")
    assert np.allclose(got[..., :3], z.real, atol=1e-14) and np.allclose(got[..., 3:], z.imag, atol=1e-14)


def test_oracle_scales_and_places():
    assert [O.pow2_scale(a) for a in (448.0, 448.1, 224.0, 1.75, 1.76, 3.5)] == [1.0, 2.0, 0.5, 2.0 ** -8, 2.0 ** -7, 2.0 ** -7]
    assert O.pow2_scale(0.0) == O.pow2_scale(1e-20) == 2.0 ** -40
    assert O.new_row_places([0, 2, 2, 5], [7, 3, 2]) == [(0, 5), (0, 6), (2, -1), (2, 0), (2, 1)]


def test_oracle_append_grows_a_page_and_starts_the_next():
    """Two calls of one row each, worked by hand: the second row quadruples the page's scale, the first row's codes move down by
    two binades; a row at a page's position 0 forgets the old scale."""
    codes, scale = np.full((8, 1, 2), 0x55, np.uint8), np.full((2, 1), 64.0, np.float32)
    table = np.array([[1, 0]])
    codes, scale = O.append_pages_e4m3(np.array([[[448.0, 1.0]]]), codes, scale, [0, 1], [1], table, 4)
    assert scale.tolist() == [[64.0], [1.0]] and O.e4m3_decode(codes[4, 0]).tolist() == [448.0, 1.0]
    codes, scale = O.append_pages_e4m3(np.array([[[-1792.0, 3.0]]]), codes, scale, [0, 1], [2], table, 4)
    assert scale.tolist() == [[64.0], [4.0]]
    assert (O.e4m3_decode(codes[4:6, 0]) * 4).tolist() == [[448.0, 1.0], [-1792.0, 3.0]]
    codes, scale = O.append_pages_e4m3(np.array([[[1.0, 2.0]]]), codes, scale, [0, 1], [5], table, 4)
    assert scale.tolist() == [[2.0 ** -7], [4.0]] and (O.e4m3_decode(codes[0, 0]) * 2.0 ** -7).tolist() == [1.0, 2.0]
    assert (codes[1:4] == 0x55).all() and (codes[6:] == 0x55).all()


def test_two_terms_keep_a_bf16_value():
    """Every bf16 significand is the sum of two E4M3 codes, hi nearest and lo the nearest to the rest, as long as lo is no
    subnormal; and a weight cut into hi and 16 lo is off by 2^-9 of itself at most."""
    x = np.concatenate([np.ldexp(1 + np.arange(128) / 128.0, e) for e in range(1, 8)] + [np.ldexp(1 + np.arange(97) / 128.0, 8)])
    assert (x <= 448).all()
    hi = O.e4m3_decode(O.e4m3_encode(x.astype(np.float32)))
    lo = O.e4m3_decode(O.e4m3_encode((x - hi).astype(np.float32)))
    assert np.array_equal(hi + lo, x)
    w = np.exp2(np.random.default_rng(1).uniform(-5, math.log2(430), size=20000)).astype(np.float32)
    hi = O.e4m3_decode(O.e4m3_encode(w))
    lo = O.e4m3_decode(O.e4m3_encode(((w - hi) * 16).astype(np.float32))) / 16
    assert (np.abs(hi + lo - w) <= 2.0 ** -9 * w).all()
    small = np.exp2(np.random.default_rng(2).uniform(-30, -5, size=20000)).astype(np.float32)
    hi = O.e4m3_decode(O.e4m3_encode(small))
    lo = O.e4m3_decode(O.e4m3_encode(((small - hi) * 16).astype(np.float32))) / 16
    assert (np.abs(hi + lo - small) <= np.maximum(2.0 ** -14, 2.0 ** -9 * small)).all()


def test_the_binding_refuses_what_is_not_on_the_gpu():
    """The argument checks run in the binding's own module, whose messages name the call and the tensor."""
    d = B.make_dims(128, 8, 128, 512, 64)
    c = torch.zeros(1, 512, dtype=torch.bfloat16)
    with pytest.raises(B.GqlaError, match="gqla_append_rope_fp8: c: expected a CUDA tensor"):
        B.gqla_append_rope_fp8(d, c, None, None, None, None, "pairs", None, None, None, 16)
    with pytest.raises(B.GqlaError, match="gqla_decode_gqa_fp8_paged: q: expected a tensor, got None"):
        B.gqla_decode_gqa_fp8_paged(d, None, c, c, c, c, c, c, c, 16, c, 1.0, 1, c, c)
    with pytest.raises(B.GqlaError, match="q_hat: expected a tensor, got list"):
        B.gqla_decode_absorb_fp8_paged(d, [1], c, c, c, 16, c, 1.0, 1, c, c)
    with pytest.raises(B.GqlaError, match="dims"):
        B.gqla_append_rope(bytearray(8), c, None, None, None, None, "pairs", None, None)
    with pytest.raises(B.GqlaError, match="style"):
        B.gqla_append_rope(d, c, None, None, None, None, "half", None, None)
