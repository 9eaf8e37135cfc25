"""Operators of a served cache: appending a step's or a prompt's rows to it with the position rotation applied on the
way (bf16 rows; E4M3 rows with a scale for every page and head), and the attention of both decoding paths over the E4M3
pages.

Dimensions are the canonical (h_q, g, d_h, r_kv, d_h^R) = (128, 8, 128, 512, 64) and the LLaMA-3-8B-shaped h_q = 32;
`draw` adds 64 heads and the 28 heads in 4 groups of the parity tests.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D_H, R_KV, D_R = 128, 512, 64
W_LATENT = R_KV + D_R
SCALE = 1.0 / math.sqrt(D_H + D_R)
TILE = 128            # rows the balanced plan counts in
SMALLEST_EXP = -40    # exponent of the smallest page scale
SPARE_PAGES = 3       # pages of the pool that no sequence owns


def _case(name, kind, h_q, batch, s_q, t_lo, t_hi, page, g=8, style="pairs"):
    """s_q = 0: a prompt, all of whose rows are new."""
    c = {"kind": kind, "h_q": h_q, "g": g, "batch": batch, "s_q": s_q, "t_lo": t_lo, "t_hi": t_hi, "page": page, "style": style}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one user's chat: the step's single new row and its queries, all latency
        _case("append_one", "append", 128, 1, 1, 777, 777, 64),
        # ragged prompts written to a bf16 cache behind their prefill
        _case("append_prompts", "append", 128, 24, 0, 100, 4000, 64, style="halves"),
        # a serving batch's step with two draft tokens over an E4M3 latent cache, partly filled pages among the touched ones
        _case("latent8_step", "latent8", 128, 64, 2, 1000, 4096, 64),
        # ragged prompts written to the E4M3 latent cache
        _case("latent8_prompts", "latent8", 128, 24, 0, 100, 4000, 64),
        # a serving batch's step on the GQA path's E4M3 planes: a scale for every page and group
        _case("planes8_step", "planes8", 32, 64, 1, 500, 3000, 32, style="halves"),
        # prompts whose expanded rows go to the planes
        _case("planes8_prompts", "planes8", 128, 16, 0, 500, 2000, 64),
        # one user's chat, absorb path: all latency
        _case("absorb8_one", "absorb8", 128, 1, 1, 777, 777, 64),
        # a full serving batch on the canonical shape (bench.py's workload) over E4M3 pages
        _case("absorb8_batch", "absorb8", 128, 64, 1, 4096, 4096, 64),
        # LLaMA-3-8B-shaped conversion, large ragged batch
        _case("absorb8_llama", "absorb8", 32, 128, 1, 512, 16384, 128),
        # one user's chat on the GQA path
        _case("gqa8_one", "gqa8", 128, 1, 1, 3001, 3001, 16),
        # the serving batch on the GQA path with multi-token prediction
        _case("gqa8_batch_mtp", "gqa8", 128, 64, 2, 4096, 4096, 64),
        # LLaMA-3-8B-shaped on the GQA path, ragged
        _case("gqa8_llama", "gqa8", 32, 64, 1, 512, 16384, 32),
    ]


def _log_int(rng: random.Random, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(("append", "latent8", "planes8", "absorb8", "absorb8", "gqa8", "gqa8"))
    h_q, g = rng.choice(((128, 8), (128, 8), (64, 8), (32, 8), (28, 4)))
    page = rng.choice((16, 32, 64, 64, 128, 256))
    step = kind in ("absorb8", "gqa8") or rng.random() < 0.5
    s_q = rng.choice((1, 1, 2, 3)) if step else 0
    rows = {"absorb8": 1 << 18, "gqa8": 1 << 18, "append": 1 << 15, "latent8": 1 << 15, "planes8": 1 << 14}[kind]
    if kind in ("append", "latent8", "planes8") and step:
        rows = 1 << 18 if kind != "planes8" else 1 << 17
    t_hi = _log_int(rng, 5, min(65536, rows))
    batch = _log_int(rng, 1, max(1, min(128, rows // t_hi)))
    t_lo = t_hi if rng.random() < 0.3 else max(1, s_q, t_hi // rng.choice((2, 8, 64)))
    return _case("", kind, h_q, batch, s_q, t_lo, t_hi, page, g, rng.choice(("pairs", "halves")))


def _lengths(case):
    """The batch's lengths are the case's own: every seed draws other values for the same batch."""
    rng = random.Random("%d %d %d" % (case["batch"], case["t_lo"], case["t_hi"]))
    return [rng.randint(case["t_lo"], case["t_hi"]) for _ in range(case["batch"])]


def _new_rows(case, lens):
    return [case["s_q"] or t for t in lens]


def _pages_of(t, page):
    return -(-t // page)


# ------------------------------------------------------------------ inputs


def _page_scale(amax):
    """The smallest power of two s with amax <= 448 s, at least 2^SMALLEST_EXP."""
    m, e = torch.frexp(amax.float())  # amax = m 2^e, 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.ldexp(torch.ones_like(m), torch.where(amax > 0, e, SMALLEST_EXP).clamp(min=SMALLEST_EXP))


def _encode(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _pool(gen, n_pages, page, heads, width, mul):
    """Pages in use: N(0, mul^2) rows, codes [pages * page, heads, width] and a scale per page and head."""
    codes = torch.empty((n_pages * page, heads, width), dtype=torch.uint8, device="cuda")
    scale = torch.empty((n_pages, heads), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 26) // (page * heads * width))
    for lo in range(0, n_pages, step):
        n = min(step, n_pages - lo)
        x = torch.randn((n, page, heads, width), generator=gen, device="cuda") * mul
        s = _page_scale(x.abs().amax(dim=(1, 3)))
        scale[lo:lo + n] = s
        codes[lo * page:(lo + n) * page] = _encode(x / s[:, None, :, None]).view(n * page, heads, width)
    return codes, scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens, page, kind = _lengths(case), case["page"], case["kind"]
    h, g, b = case["h_q"], case["g"], case["batch"]
    counts = [_pages_of(t, page) for t in lens]
    n_pages = sum(counts) + SPARE_PAGES
    order = list(range(n_pages))
    random.Random(seed + 1).shuffle(order)
    table = torch.zeros((b, max(counts)), dtype=torch.int32)
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)

    state = {"case": dict(case), "table": table.cuda(), "seqlens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
             "max_len": max(lens)}
    if kind in ("absorb8", "gqa8"):
        q_width = W_LATENT if kind == "absorb8" else D_H + D_R
        state["q"] = normal(b, case["s_q"], h, q_width)
        if kind == "absorb8":
            # a latent query is a sum over d_h products: its scores with unit-variance rows stay of the order of one
            state["q"].mul_(math.sqrt((D_H + D_R) / W_LATENT))
            codes, scale = _pool(gen, n_pages, page, 1, W_LATENT, 1.0)
            state["cache8"], state["page_scale"] = codes.view(-1, W_LATENT), scale.view(-1)
        else:
            state["k_c8"], state["k_scale"] = _pool(gen, n_pages, page, g, D_H, 1.0)
            state["v8"], state["v_scale"] = _pool(gen, n_pages, page, g, D_H, 0.5)
            codes, scale = _pool(gen, n_pages, page, 1, D_R, 1.0)
            state["k_r8"], state["r_scale"] = codes.view(-1, D_R), scale.view(-1)
        return state
    new = _new_rows(case, lens)
    n = sum(new)
    starts = [0]
    for k in new:
        starts.append(starts[-1] + k)
    state["new_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    state["k_r"] = normal(n, D_R)
    freq = 10000.0 ** (-torch.arange(0, D_R, 2, dtype=torch.float64, device="cuda") / D_R)
    angle = torch.arange(max(lens), dtype=torch.float64, device="cuda")[:, None] * freq
    state["rope"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    if case["s_q"]:  # a step's queries are rotated along with its keys; a prompt's belong to its prefill
        state["q_r"] = normal(n, h, D_R)
        state["q_out"] = torch.empty_like(state["q_r"])
    if kind == "planes8":
        state["k_c"], state["v"] = normal(n, g, D_H), normal(n, g, D_H).mul_(0.5)
        state["k_c8"], state["k_scale"] = _pool(gen, n_pages, page, g, D_H, 1.0)
        state["v8"], state["v_scale"] = _pool(gen, n_pages, page, g, D_H, 0.5)
        codes, scale = _pool(gen, n_pages, page, 1, D_R, 1.0)
        state["k_r8"], state["r_scale"] = codes.view(-1, D_R), scale.view(-1)
        return state
    state["c"] = normal(n, R_KV)
    if kind == "append":
        state["cache"] = normal(n_pages * page, W_LATENT)
    else:
        codes, scale = _pool(gen, n_pages, page, 1, W_LATENT, 1.0)
        state["cache8"], state["page_scale"] = codes.view(-1, W_LATENT), scale.view(-1)
    return state


# ------------------------------------------------------------------ plain forms


def _positions(state):
    """Sequence and position of every new row; the rows are packed, sequence 0 first."""
    start = state["new_start"].long()
    n = state["k_r"].shape[0]
    count = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count, output_size=n)
    pos = state["seqlens"].long()[seq] - count[seq] + torch.arange(n, device="cuda") - start[seq]
    return seq, pos


def _rotated(x, rope, pos, style):
    """x [N, ..., d]: the pairs of `style` turned by the angles of the rows' positions, in 32 bits."""
    d = x.shape[-1]
    cos, sin = (rope[pos][:, o:o + d // 2].view(-1, *([1] * (x.dim() - 2)), d // 2) for o in (0, d // 2))
    x = x.float()
    if style == "pairs":
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)


def _plain_append8(state, seq, pos, rows, codes, scale):
    """rows [N, H, W] into codes [pool rows, H, W] with scale [pages, H]: a page keeps the largest scale that its rows
    have needed; its older rows are coded anew when it grows."""
    page, table = state["case"]["page"], state["table"].long()
    n, heads = rows.shape[:2]
    pid = table[seq, pos // page]
    amax = torch.zeros_like(scale).scatter_reduce_(0, pid[:, None].expand(n, heads), rows.abs().amax(-1), "amax")
    touched = torch.zeros(scale.shape[0], dtype=torch.bool, device="cuda")
    touched[pid] = True
    first = pos[state["new_start"][:-1].long()]
    first_pid = table[torch.arange(table.shape[0], device="cuda"), first // page]
    older = first % page
    before = scale[first_pid]
    floor = torch.zeros_like(scale)
    floor[first_pid] = torch.where((older > 0)[:, None], before, 0.0)
    scale.copy_(torch.where(touched[:, None], torch.maximum(_page_scale(amax), floor), scale))
    at = first_pid[:, None] * page + torch.arange(page, device="cuda")
    kept = codes[at]  # [B, page, H, W]
    again = _encode(_decode(kept) * (before / scale[first_pid])[:, None, :, None])
    codes[at] = torch.where((torch.arange(page, device="cuda") < older[:, None])[:, :, None, None], again, kept)
    codes[pid * page + pos % page] = _encode(rows / scale[pid][:, :, None])


def _paged_rows(state, codes, scale):
    """Rows [B, max_len, H, W] in 32 bits (behind a sequence's end: anything, masked by the caller)."""
    page = state["case"]["page"]
    t = torch.arange(state["max_len"], device="cuda")
    pid = state["table"].long()[:, t // page]
    return _decode(codes[pid * page + t % page]) * scale[pid][..., None]


def _plain_attention(state, q, k, v):
    """q [B, s, G, P, W], k [B, T, G, W], v [B, T, G, V]: causal within the step, in 32 bits."""
    b, s = q.shape[:2]
    scores = torch.einsum("bsgpw,btgw->bsgpt", q, k) * SCALE
    seen = state["seqlens"].long()[:, None] - (s - 1 - torch.arange(s, device="cuda"))
    hidden = torch.arange(k.shape[1], device="cuda") >= seen[:, :, None]
    scores = scores.masked_fill_(hidden[:, :, None, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    prob = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = prob.sum(-1, keepdim=True)
    o = torch.einsum("bsgpt,btgv->bsgpv", prob, v) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    return o.reshape(b, s, -1, v.shape[-1]).to(torch.bfloat16), lse.reshape(b, s, -1)


def _plain(state):
    case = state["case"]
    kind, g = case["kind"], case["g"]
    if kind == "absorb8":
        rows = _paged_rows(state, state["cache8"][:, None], state["page_scale"][:, None])
        return _plain_attention(state, state["q"].float()[:, :, None], rows, rows[..., :R_KV])
    if kind == "gqa8":
        q = state["q"].float()
        k_r = _paged_rows(state, state["k_r8"][:, None], state["r_scale"][:, None])
        k = torch.cat([_paged_rows(state, state["k_c8"], state["k_scale"]), k_r.expand(-1, -1, g, -1)], dim=-1)
        v = _paged_rows(state, state["v8"], state["v_scale"])
        return _plain_attention(state, q.view(*q.shape[:2], g, -1, q.shape[-1]), k, v)
    seq, pos = _positions(state)
    k_r = _rotated(state["k_r"], state["rope"], pos, case["style"])
    if "q_r" in state:
        state["q_out"].copy_(_rotated(state["q_r"], state["rope"], pos, case["style"]))
    if kind == "planes8":
        _plain_append8(state, seq, pos, state["k_c"].float(), state["k_c8"], state["k_scale"])
        _plain_append8(state, seq, pos, state["v"].float(), state["v8"], state["v_scale"])
        _plain_append8(state, seq, pos, k_r[:, None], state["k_r8"][:, None], state["r_scale"][:, None])
        return _appended(state)
    rows = torch.cat([state["c"].float(), k_r], dim=-1)
    if kind == "latent8":
        _plain_append8(state, seq, pos, rows[:, None], state["cache8"][:, None], state["page_scale"][:, None])
    else:
        page = case["page"]
        slot = state["table"].long()[seq, pos // page] * page + pos % page
        state["cache"][slot] = rows.to(torch.bfloat16)
    return _appended(state)


def _appended(state):
    out = {k: state[k] for k in ("q_out", "cache", "page_scale", "k_scale", "v_scale", "r_scale") if k in state}
    out |= {k: state[k].view(torch.float8_e4m3fn) for k in ("cache8", "k_c8", "v8", "k_r8") if k in state}
    return out


# ------------------------------------------------------------------ the framework's calls


def _own(state):
    from paper_2605_15250_b200 import binding as B

    case = state["case"]
    kind, page = case["kind"], case["page"]
    if "dims" not in state:  # what a decoder keeps from step to step: the shape, the plan and its workspaces
        state["dims"] = B.make_dims(case["h_q"], case["g"], D_H, R_KV, D_R)
        if kind in ("absorb8", "gqa8"):
            b, s, h = state["q"].shape[:3]
            lens = _lengths(case)
            path, width = ("absorb", R_KV) if kind == "absorb8" else ("gqa", D_H)
            workers = B.gqla_fp8_paged_workers(state["dims"], torch.bfloat16, s, page, path)
            tiles = [-(-t // TILE) for t in lens]
            share = max(1, -(-sum(tiles) // max(workers, 1)))
            slots = -(-max(tiles) // share) + 1
            state["splits"] = -slots
            state["o_part"] = torch.empty((b, slots, s, h, width), dtype=torch.float32, device="cuda")
            state["lse_part"] = torch.empty((b, slots, s, h), dtype=torch.float32, device="cuda")
            state["out"] = torch.empty((b, s, h, width), dtype=torch.bfloat16, device="cuda")
            state["lse"] = torch.empty((b, s, h), dtype=torch.float32, device="cuda")
    dims = state["dims"]
    if kind == "absorb8":
        B.gqla_decode_absorb_fp8_paged(dims, state["q"], state["cache8"], state["page_scale"], state["table"], page,
                                       state["seqlens"], SCALE, state["splits"], state["o_part"], state["lse_part"],
                                       state["out"], state["lse"])
        return state["out"], state["lse"]
    if kind == "gqa8":
        B.gqla_decode_gqa_fp8_paged(dims, state["q"], state["k_c8"], state["v8"], state["k_r8"], state["k_scale"],
                                    state["v_scale"], state["r_scale"], state["table"], page, state["seqlens"], SCALE,
                                    state["splits"], state["o_part"], state["lse_part"], state["out"], state["lse"])
        return state["out"], state["lse"]
    step = (state["new_start"], state["seqlens"])
    turn = (state["rope"], case["style"])
    queries = (state.get("q_r"), state.get("q_out"))
    if kind == "append":
        B.gqla_append_rope(dims, state["c"], state["k_r"], *step, *turn, state["cache"], None, state["table"], page, *queries)
    elif kind == "latent8":
        B.gqla_append_rope_fp8(dims, state["c"], state["k_r"], *step, *turn, state["cache8"], state["page_scale"],
                               state["table"], page, *queries)
    else:
        B.gqla_append_planes_fp8(dims, state["k_c"], state["v"], state["k_r"], *step, *turn, state["k_c8"], state["v8"],
                                 state["k_r8"], state["k_scale"], state["v_scale"], state["r_scale"], state["table"], page,
                                 *queries)
    return _appended(state)


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Every new row, query, weight-free table row and cache row once; the products of Eqs. (mqa) and (mha)."""
    lens, page, kind = _lengths(case), case["page"], case["kind"]
    h, g = case["h_q"], case["g"]
    pages = sum(_pages_of(t, page) for t in lens)
    ints = 4 * (pages + 2 * len(lens))
    if kind in ("absorb8", "gqa8"):
        rows, n_q = sum(lens), case["batch"] * case["s_q"] * h
        seen = rows * h * case["s_q"]
        if kind == "absorb8":
            return {"bytes": rows * W_LATENT + 4 * pages + ints + n_q * (2 * W_LATENT + 2 * R_KV + 4),
                    "flops": 2.0 * seen * (2 * R_KV + D_R)}
        return {"bytes": rows * (2 * g * D_H + D_R) + 4 * pages * (2 * g + 1) + ints + n_q * (2 * (2 * D_H + D_R) + 4),
                "flops": 2.0 * seen * (2 * D_H + D_R)}
    new = _new_rows(case, lens)
    n = sum(new)
    touched = sum(_pages_of(t, page) - (t - k) // page for t, k in zip(lens, new))
    turned = n * D_R * (1 + (h if case["s_q"] else 0))
    width = 2 * g * D_H + D_R if kind == "planes8" else W_LATENT
    heads = {"append": 0, "latent8": 1, "planes8": 2 * g + 1}[kind]
    positions = len(set(p for t, k in zip(lens, new) for p in range(t - k, t)))
    return {"bytes": n * width * (4 if kind == "append" else 3) + 4 * positions * D_R + 4 * touched * (1 + heads) + 8 * len(lens)
            + (4 * n * h * D_R if case["s_q"] else 0), "flops": 3.0 * turned}


# ------------------------------------------------------------------ the definition, in 64 bits


def _exact_rotation(x, pos, table, style):
    """Rows x [n, ..., d] turned one pair at a time: (a + i b) times e^(i angle), as complex numbers."""
    d = x.shape[-1]
    x = x.double()
    z = torch.complex(x[..., 0::2], x[..., 1::2]) if style == "pairs" else torch.complex(x[..., :d // 2], x[..., d // 2:])
    t = table.double()[pos]
    z = z * torch.complex(t[:, :d // 2], t[:, d // 2:]).view(len(pos), *([1] * (x.dim() - 2)), d // 2)
    return torch.view_as_real(z).flatten(-2) if style == "pairs" else torch.cat([z.real, z.imag], dim=-1)


def _exact_code(x):
    """Nearest E4M3 value, ties to the even one, at most 448: spacing 2^(e - 3) in the binade of 2^e, 2^-9 below 2^-6."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    unit = torch.exp2(e - 3)
    return (torch.round(x / unit) * unit).clamp(-448.0, 448.0)


def _exact_scale(amax):
    e = math.ceil(math.log2(amax / 448.0)) if amax > 0 else SMALLEST_EXP
    while amax > 448.0 * 2.0 ** e:
        e += 1
    while e > SMALLEST_EXP and amax <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** max(e, SMALLEST_EXP)


def _exact_append8(case, table, lens, new, rows, codes, scale):
    """One page after the other; rows [N, H, W] in 64 bits, codes (values) and scale are changed in place."""
    page, at = case["page"], 0
    for b, (t, k) in enumerate(zip(lens, new)):
        for p0 in range((t - k) // page * page, t, page):
            lo, hi = max(p0, t - k), min(p0 + page, t)
            pid = table[b][p0 // page]
            mine = rows[at + lo - (t - k):at + hi - (t - k)]
            amax = mine.abs().amax(dim=(0, 2)).tolist()
            for head, a in enumerate(amax):
                s = _exact_scale(a)
                if lo > p0:
                    was = float(scale[pid, head])
                    if was >= s:
                        s = was
                    else:
                        old = codes[pid * page:pid * page + lo - p0, head]
                        codes[pid * page:pid * page + lo - p0, head] = _exact_code(old * (was / s))
                scale[pid, head] = s
                codes[pid * page + lo - p0:pid * page + hi - p0, head] = _exact_code(mine[:, head] / s)
        at += k


def exact(case, seed):
    state = prepare(case, seed)
    lens, page, kind, g = _lengths(case), case["page"], case["kind"], case["g"]
    table = state["table"].tolist()
    if kind in ("absorb8", "gqa8"):
        q = state["q"].double()
        b, s, h = q.shape[:3]
        out = torch.zeros((b, s, h, R_KV if kind == "absorb8" else D_H), dtype=torch.float64, device="cuda")
        lse = torch.full((b, s, h), -math.inf, dtype=torch.float64, device="cuda")

        def plane(codes, scale, seq):
            ids = torch.tensor(table[seq][:_pages_of(lens[seq], page)], device="cuda")
            vals = codes.view(torch.float8_e4m3fn).view(-1, page, *codes.shape[1:])[ids].double()
            vals = vals * scale[ids].double().view(len(ids), 1, *scale.shape[1:], 1)
            return vals.flatten(0, 1)[:lens[seq]]

        for i in range(b):
            if kind == "absorb8":
                k = plane(state["cache8"], state["page_scale"], i)
                x = torch.einsum("shw,tw->sht", q[i], k)
            else:
                k_c, v = plane(state["k_c8"], state["k_scale"], i), plane(state["v8"], state["v_scale"], i)
                k_r = plane(state["k_r8"], state["r_scale"], i)
                x = (torch.einsum("sgpw,tgw->sgpt", q[i, ..., :D_H].reshape(s, g, h // g, D_H), k_c).reshape(s, h, -1)
                     + torch.einsum("shw,tw->sht", q[i, ..., D_H:], k_r))
            x = x * SCALE
            for p in range(s):
                n = lens[i] - (s - 1 - p)
                if n <= 0:
                    continue
                w = torch.softmax(x[p, :, :n], dim=-1)
                lse[i, p] = torch.logsumexp(x[p, :, :n], dim=-1)
                out[i, p] = w @ k[:n, :R_KV] if kind == "absorb8" else torch.einsum(
                    "gpt,tgv->gpv", w.view(g, h // g, n), v[:n]).reshape(h, D_H)
        return out, lse
    new = _new_rows(case, lens)
    pos = torch.tensor([p for t, k in zip(lens, new) for p in range(t - k, t)], device="cuda")
    k_r = _exact_rotation(state["k_r"], pos, state["rope"], case["style"])
    out = {}
    if case["s_q"]:
        out["q_out"] = _exact_rotation(state["q_r"], pos, state["rope"], case["style"])
    if kind == "append":
        cache = state["cache"].double()
        slots = torch.tensor([table[b][p // page] * page + p % page for b, (t, k) in enumerate(zip(lens, new))
                              for p in range(t - k, t)], device="cuda")
        cache[slots] = torch.cat([state["c"].double(), k_r], dim=-1)
        return out | {"cache": cache}
    if kind == "latent8":
        todo = [("cache8", "page_scale", torch.cat([state["c"].double(), k_r], dim=-1)[:, None])]
    else:
        todo = [("k_c8", "k_scale", state["k_c"].double()), ("v8", "v_scale", state["v"].double()), ("k_r8", "r_scale", k_r[:, None])]
    for name, scale_name, rows in todo:
        codes = state[name].view(torch.float8_e4m3fn).double()
        scale = state[scale_name].double()
        _exact_append8(case, table, lens, new, rows, codes.view(codes.shape[0], rows.shape[1], -1), scale.view(scale.shape[0], -1))
        out[name], out[scale_name] = codes, scale
    return out
