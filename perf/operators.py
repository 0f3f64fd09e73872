"""The operators of a decode step on a paged key-value cache: what is measured.

Five operators, in the order in which a serving step of several requests calls
them:

  plan    block tables, slot maps and positions of the rows that a step adds,
          built from the requests' lengths and the list of free pages
  append  the new key and value rows stored into their pages
  attn    attention of one new token per request over its pages, the hidden
          (visual) block of a request left out
  norm    residual addition, RMSNorm with a weight, and the normalised row also
          in 8 bits (e4m3) with one scale per row
  w4      few rows times a matrix of 4-bit weights with group scales, rows in
          bf16 or in the 8 bits that the norm writes

Where `own` is false, run() computes the plain form in elementary torch
operations in 32 bits. Layer shapes are the repository's own (hidden 2048, 32
query heads on 4 KV heads of 128, the 2049 rows of the text-only cache, 1552
rows, 16384 rows) or generic.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
SCRATCH = 16 << 20  # bytes of workspace that a serving program keeps for the attention


def listed():
    return [
        # The slots of one decode step: a batch of 24 requests adds one row each.
        {"name": "plan_decode_B24", "kind": "plan", "B": 24, "ps": 16, "lo": 1, "hi": 4096, "fresh": 1, "chunks": 0,
         "chunk": 0},
        # A mixed step of a busy server: 509 requests add one row each and 11
        # prompts come in with 1552 rows.
        {"name": "plan_mixed_B520", "kind": "plan", "B": 520, "ps": 64, "lo": 1, "hi": 16385, "fresh": 1,
         "chunks": 11, "chunk": 1552},
        # One layer's new rows of a decode batch of odd size.
        {"name": "append_decode_N23", "kind": "append", "N": 23, "hkv": 4, "d": 128, "ps": 16, "pages": 2000},
        # One layer's rows of the longest prompt, stored into its pages.
        {"name": "append_prompt_N16384", "kind": "append", "N": 16384, "hkv": 4, "d": 128, "ps": 64, "pages": 600},
        # One request over the text-only cache: the latency of a decode step.
        {"name": "attn_B1_C2049", "kind": "attn", "B": 1, "lo": 2049, "hi": 2049, "hide": 0.0, "hq": 32, "hkv": 4,
         "d": 128, "ps": 16, "empty": 0},
        # A full batch of long multimodal requests after the exit, their visual
        # blocks hidden: the largest call.
        {"name": "attn_B96_ragged", "kind": "attn", "B": 96, "lo": 2000, "hi": 16385, "hide": 0.6, "hq": 32, "hkv": 4,
         "d": 128, "ps": 64, "empty": 0},
        # Many short chats on a small model: heads of 64, a KV head for every
        # query head, and two slots of the batch without a request.
        {"name": "attn_B97_D64", "kind": "attn", "B": 97, "lo": 5, "hi": 1553, "hide": 0.0, "hq": 16, "hkv": 16,
         "d": 64, "ps": 32, "empty": 2},
        # The norm in front of a decode batch's projections.
        {"name": "norm_T24", "kind": "norm", "T": 24, "d": 2048, "dtype": "bf16"},
        # The norm of the longest prompt.
        {"name": "norm_T16384", "kind": "norm", "T": 16384, "d": 2048, "dtype": "bf16"},
        # Query, key and value projections of one token, from the norm's 8 bits.
        {"name": "w4_qkv_T1", "kind": "w4", "T": 1, "n": 5120, "k": 2048, "group": 128, "x": "e4m3"},
        # Output projection of a decode batch, from the attention's rows.
        {"name": "w4_out_T17", "kind": "w4", "T": 17, "n": 2048, "k": 4096, "group": 64, "x": "bf16"},
        # A large projection (a wide model's, or a vocabulary's), small batch.
        {"name": "w4_wide_T8", "kind": "w4", "T": 8, "n": 32001, "k": 8192, "group": 128, "x": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _step(rng, lo, hi, granule):
    """A multiple of granule: an odd one, or a power of two times it."""
    v = max(1, _log(rng, lo, hi) // granule)
    return granule * (1 << (v.bit_length() - 1) if rng.random() < 0.5 else v | 1)


def draw(rng):
    kind = rng.choice(["plan", "append", "attn", "attn", "norm", "w4", "w4"])
    if kind == "plan":
        hi = _log(rng, 16, 16385)
        return {"kind": "plan", "B": _log(rng, 1, 600), "ps": rng.choice([8, 16, 32, 64, 128]),
                "lo": rng.choice([0, 1, 16]), "hi": hi, "fresh": rng.choice([0, 1, 1, 4]),
                "chunks": rng.choice([0, 0, 1, 3, 9]), "chunk": _log(rng, 17, 1801)}
    if kind == "append":
        d = rng.choice([64, 128])
        hkv = rng.choice([1, 2, 4, 8])
        ps = rng.choice([8, 16, 32, 64, 128])
        N = _log(rng, 1, 16000 * 4 // (8 if hkv == 8 else 4))
        return {"kind": "append", "N": N, "hkv": hkv, "d": d, "ps": ps, "pages": (2 * N + 999) // ps + 1}
    if kind == "attn":
        hkv, per = rng.choice([(1, 8), (4, 8), (4, 8), (8, 4), (2, 16), (8, 1), (4, 6), (5, 5)])
        d = rng.choice([64, 128, 128])
        # keys in all, by the bytes that the largest listed case reads
        most = 250_000 * 512 // (hkv * d)
        hi = _log(rng, 3, 40_000)
        B = min(_log(rng, 1, 200), max(1, most // hi))
        lo = rng.choice([1, max(1, hi // 8), hi])
        return {"kind": "attn", "B": B, "lo": lo, "hi": hi, "hide": rng.choice([0.0, 0.0, 0.5, 0.9]), "hq": hkv * per,
                "hkv": hkv, "d": d, "ps": rng.choice([8, 16, 32, 64, 128]), "empty": rng.choice([0, 0, 1]) if B > 1 else 0}
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = _step(rng, 64, 8192, 64)
        T = min(_log(rng, 1, 16000), 33_000_000 // d // (2 if dtype == "f32" else 1))
        return {"kind": "norm", "T": T, "d": d, "dtype": dtype}
    group = rng.choice([32, 64, 128, 128])
    k = _step(rng, 256, 8192, group)
    n = _log(rng, 64, min(32000, 250_000_000 // k))
    return {"kind": "w4", "T": rng.choice([1, 1, 2, 5, 8, 13, 24, 32]), "n": n, "k": k, "group": group,
            "x": rng.choice(["bf16", "e4m3"])}


# ------------------------------------------------------------------ inputs

def _lengths(c):
    """The requests' lengths: spread evenly over the logarithm of [lo, hi]."""
    lo, hi, B = c["lo"], c["hi"], c["B"]
    a, b = math.log(lo + 1.0), math.log(hi + 1.0)
    return [int(round(math.exp(a + (b - a) * (i + 1) / B))) - 1 for i in range(B)]


def _hidden(c, n):
    """(begin, count) of the hidden block of a request of n rows."""
    return (min(16, n // 8), int(n * c["hide"])) if c["hide"] else (0, 0)


def _attn_lengths(c):
    n = _lengths(c)
    return [0] * c["empty"] + n[c["empty"]:]


def _fresh(c):
    """New rows of each request: `fresh`, or `chunk` for the first `chunks` of them."""
    return [c["chunk"] if i < c["chunks"] else c["fresh"] for i in range(c["B"])]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 13)
    return _PREPARE[case["kind"]](case, g)


def _prepare_plan(c, g):
    B, ps = c["B"], c["ps"]
    order = torch.randperm(B, generator=g, device=DEV)
    cached = _i32(_lengths(c))[order]
    fresh = _i32(_fresh(c))[torch.randperm(B, generator=g, device=DEV)]
    have, need = -(-cached // ps), -(-(cached + fresh) // ps)
    width = -(-(max(_lengths(c)) + max(_fresh(c))) // ps) + 3
    held, new = sum(-(-n // ps) for n in _lengths(c)), sum(-(-n // ps) + 1 for n in _fresh(c))
    pages = torch.randperm(held + new + 5, generator=g, device=DEV).to(torch.int32)
    cols = torch.arange(width, device=DEV)[None]
    start = (torch.cumsum(have, 0) - have)[:, None]
    table = torch.where(cols < have[:, None], pages[(start + cols).clamp(max=held + new)], -1).to(torch.int32)
    n = sum(_fresh(c))
    rows = n + 7  # the slot map of a step is padded to the size that the step was captured for
    e = lambda m: torch.empty(m, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"case": c, "cached": cached, "fresh": fresh, "free": pages[held:].contiguous(), "table": table,
            "head": _i32([2]), "head_out": e(1), "seq_len": e(B), "row_start": e(B + 1), "slots": e(rows),
            "positions": e(rows), "status": torch.zeros(1, dtype=torch.int32, device=DEV)}


def _prepare_append(c, g):
    N, hkv, d, ps, P = c["N"], c["hkv"], c["d"], c["ps"], c["pages"]
    # the rows as a fused projection leaves them: keys and values inside wider rows
    qkv = torch.randn(N, 4 * hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    slots = torch.randperm(P * ps, generator=g, device=DEV)[:N].to(torch.int32)
    if N > 3:
        slots[torch.randint(0, N, (1,), generator=g, device=DEV)] = -1  # a padded row
    kp, vp = (torch.randn(P, ps, hkv, d, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    return {"case": c, "k": qkv[:, 2 * hkv:3 * hkv], "v": qkv[:, 3 * hkv:], "slots": slots, "kp": kp, "vp": vp}


def _prepare_attn(c, g):
    B, ps, hq, hkv, d = c["B"], c["ps"], c["hq"], c["hkv"], c["d"]
    n = _attn_lengths(c)
    order = torch.randperm(B, generator=g, device=DEV)
    hid = [_hidden(c, x) for x in n]
    lens, hb, hc = _i32(n)[order], _i32([h[0] for h in hid])[order], _i32([h[1] for h in hid])[order]
    width = max(1, -(-max(n) // ps))
    used = -(-lens // ps)
    total = sum(-(-x // ps) for x in n)
    P = total + 8
    pages = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
    cols = torch.arange(width, device=DEV)[None]
    start = (torch.cumsum(used, 0) - used)[:, None]
    # pages that lie wholly inside a hidden block have been given back
    gone = (cols * ps >= hb[:, None]) & ((cols + 1) * ps <= (hb + hc)[:, None])
    table = torch.where((cols < used[:, None]) & ~gone, pages[(start + cols).clamp(max=P - 1)], -1).to(torch.int32)
    q = torch.randn(B, hq + 2 * hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    kp, vp = (torch.empty(P, ps, hkv, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    return {"case": c, "q": q[:, :hq], "kp": kp, "vp": vp, "table": table, "lens": lens,
            "hb": hb if c["hide"] else None, "hc": hc if c["hide"] else None,
            "out": torch.empty(B, hq, d, dtype=torch.bfloat16, device=DEV),
            "ws": torch.empty(SCRATCH, dtype=torch.uint8, device=DEV)}


def _prepare_norm(c, g):
    T, d = c["T"], c["d"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    x = torch.randn(T, d, generator=g, device=DEV).to(dt)
    # the residual stream grows over the layers, a few of its features much more than the others
    r = torch.randn(T, d, generator=g, device=DEV) * 4
    r[:, :: max(1, d // 7)] *= 10
    w = (1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(dt)
    e = lambda t: torch.empty(T, d, dtype=t, device=DEV)  # noqa: E731
    return {"case": c, "x": x, "res": r.to(dt), "w": w, "sum": e(dt), "y": e(dt), "y8": e(torch.float8_e4m3fn),
            "scale": torch.empty(T, dtype=torch.float32, device=DEV)}


def _prepare_w4(c, g):
    T, n, k, group = c["T"], c["n"], c["k"], c["group"]
    w = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    ws = (torch.rand(n, k // group, generator=g, device=DEV) * 0.01 + 0.002).to(torch.bfloat16)
    x = torch.randn(T, k, generator=g, device=DEV)
    xs = None
    if c["x"] == "e4m3":
        a = x.abs().amax(1)
        x, xs = (x * (448 / a)[:, None]).to(torch.float8_e4m3fn), a / 448
    else:
        x = x.to(torch.bfloat16)
    return {"case": c, "x": x, "xs": xs, "w": w, "ws": ws,
            "out": torch.empty(T, n, dtype=torch.bfloat16, device=DEV)}


_PREPARE = {"plan": _prepare_plan, "append": _prepare_append, "attn": _prepare_attn, "norm": _prepare_norm,
            "w4": _prepare_w4}


# ------------------------------------------------------------------ the calls

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


def _own_plan(s):
    import paper_2609_38823_gb300 as dm

    dm.decomoe_paged_plan(s["cached"], s["fresh"], s["case"]["ps"], s["free"], s["table"], s["seq_len"],
                          s["row_start"], s["slots"], s["positions"], free_head=s["head"],
                          free_head_out=s["head_out"], status=s["status"])
    return {k: s[k] for k in ("table", "seq_len", "row_start", "slots", "positions", "head_out")}


def _own_append(s):
    import paper_2609_38823_gb300 as dm

    dm.decomoe_paged_append(s["k"], s["v"], s["slots"], s["kp"], s["vp"])
    return {"kp": s["kp"], "vp": s["vp"]}


def _own_attn(s):
    import paper_2609_38823_gb300 as dm

    dm.decomoe_paged_attention(s["q"], s["kp"], s["vp"], s["table"], s["lens"], s["out"], s["ws"],
                               hide_begin=s["hb"], hide_count=s["hc"])
    return s["out"]


def _own_norm(s):
    import paper_2609_38823_gb300 as dm

    dm.decomoe_add_rmsnorm_q8(s["x"], s["res"], s["w"], s["sum"], s["y"], s["y8"], s["scale"])
    return {k: s[k] for k in ("sum", "y", "y8", "scale")}


def _own_w4(s):
    import paper_2609_38823_gb300 as dm

    dm.decomoe_w4_linear(s["x"], s["w"], s["ws"], s["out"], x_scale=s["xs"])
    return s["out"]


_OWN = {"plan": _own_plan, "append": _own_append, "attn": _own_attn, "norm": _own_norm, "w4": _own_w4}


# ------------------------------------------------------------------ plain forms

def _plain_plan(s):
    ps, cached, fresh, table = s["case"]["ps"], s["cached"], s["fresh"], s["table"]
    seq_len = cached + fresh
    have, need = (cached + ps - 1) // ps, (seq_len + ps - 1) // ps
    new = need - have
    ends = torch.cumsum(new, 0)
    start = s["head"] + ends - new
    cols = torch.arange(table.shape[1], device=DEV)[None]
    at = (start[:, None] + cols - have[:, None]).clamp(0, s["free"].shape[0] - 1)
    fill = (cols >= have[:, None]) & (cols < need[:, None])
    table = torch.where(fill, s["free"][at], table)
    row_end = torch.cumsum(fresh, 0)
    row_start = torch.cat([torch.zeros_like(row_end[:1]), row_end])
    r = torch.arange(s["slots"].shape[0], device=DEV)
    b = torch.searchsorted(row_end, r, right=True)
    there = b < fresh.shape[0]
    b = b.clamp(max=fresh.shape[0] - 1)
    pos = torch.where(there, cached[b] + r - row_start[b], 0)
    slots = torch.where(there, table[b, pos // ps] * ps + pos % ps, -1)
    positions = torch.where(there, pos, -1)
    i = torch.int32
    return {"table": table, "seq_len": seq_len, "row_start": row_start.to(i), "slots": slots.to(i),
            "positions": positions.to(i), "head_out": (s["head"] + ends[-1:]).to(i)}


def _plain_append(s):
    keep = s["slots"] >= 0
    # a row without a slot stores another row's values once more in its place
    src = torch.where(keep, torch.arange(keep.shape[0], device=DEV), keep.to(torch.uint8).argmax())
    at = s["slots"][src].long()
    for pages, new in ((s["kp"], s["k"]), (s["vp"], s["v"])):
        pages.view(-1, *pages.shape[2:])[at] = new[src]
    return {"kp": s["kp"], "vp": s["vp"]}


def _plain_attn(s):
    q, table, lens = s["q"], s["table"], s["lens"]
    B, hq, d = q.shape
    hkv = s["kp"].shape[2]
    at = table.clamp(min=0).long()
    k, v = (p[at].flatten(1, 2).float() for p in (s["kp"], s["vp"]))  # [B, keys, hkv, d]
    j = torch.arange(k.shape[1], device=DEV)[None]
    see = j < lens[:, None]
    if s["hb"] is not None:
        see &= (j < s["hb"][:, None]) | (j >= (s["hb"] + s["hc"])[:, None])
    x = torch.einsum("bghd,bkgd->bghk", q.view(B, hkv, hq // hkv, d).float(), k) / math.sqrt(d)
    x = torch.where(see[:, None, None], x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0, m))
    o = torch.einsum("bghk,bkgd->bghd", p, v)
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, o / torch.where(total > 0, total, 1), 0)
    return o.reshape(B, hq, d).to(torch.bfloat16)


TINY = 2.0 ** -100  # the least row maximum that a scale is made for


def _plain_norm(s):
    x = s["x"].float() + s["res"].float()
    v = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * s["w"].float()
    a = v.abs().amax(-1, keepdim=True).clamp(min=TINY)
    dt = s["x"].dtype
    return {"sum": x.to(dt), "y": v.to(dt), "y8": (v * (448 / a)).to(torch.float8_e4m3fn), "scale": (a / 448)[:, 0]}


def _plain_w4(s):
    w, ws = s["w"], s["ws"].float()
    q = torch.stack([w & 15, w >> 4], -1).flatten(1).float() - 8
    full = (q.unflatten(1, (ws.shape[1], -1)) * ws[:, :, None]).flatten(1)
    y = s["x"].float() @ full.t()
    if s["xs"] is not None:
        y = y * s["xs"][:, None]
    return y.to(torch.bfloat16)


_PLAIN = {"plan": _plain_plan, "append": _plain_append, "attn": _plain_attn, "norm": _plain_norm, "w4": _plain_w4}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """run()'s outputs from the definitions in 64 bits, one request or row
    block at a time; None for whole-number outputs."""
    if case["kind"] == "plan":
        return None
    return _EXACT[case["kind"]](prepare(case, seed))


def _exact_append(s):
    out = {}
    for name, new in (("kp", s["k"]), ("vp", s["v"])):
        pages = s[name].double()
        ps = pages.shape[1]
        slots = s["slots"].tolist()
        rows = [r for r, x in enumerate(slots) if x >= 0]
        page, off = torch.tensor([[slots[r] // ps, slots[r] % ps] for r in rows], device=DEV).t()
        pages[page, off] = new.double()[torch.tensor(rows, device=DEV)]
        out[name] = pages
    return out


def _exact_attn(s):
    B, hq, d = s["q"].shape
    hkv, ps = s["kp"].shape[2], s["kp"].shape[1]
    out = torch.zeros(B, hq, d, dtype=torch.float64, device=DEV)
    lens = s["lens"].tolist()
    hide = [(0, 0)] * B if s["hb"] is None else list(zip(s["hb"].tolist(), s["hc"].tolist()))
    for b in range(B):
        h0, h1 = hide[b][0], hide[b][0] + hide[b][1]
        j = torch.tensor([i for i in range(lens[b]) if not h0 <= i < h1], dtype=torch.long, device=DEV)
        if not len(j):
            continue
        page, off = s["table"][b].long()[j // ps], j % ps
        k, v = s["kp"][page, off].double(), s["vp"][page, off].double()
        for h in range(hkv):
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            x = s["q"][b, heads].double() @ k[:, h].t() * d ** -0.5
            out[b, heads] = torch.softmax(x, -1) @ v[:, h]
    return out


def _exact_norm(s):
    x = s["x"].double().add_(s["res"].double())
    v = x * s["w"].double() / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[1] + 1e-6)
    scale = torch.clamp(torch.amax(torch.abs(v), -1), min=TINY) / 448
    return {"sum": x, "y": v, "y8": v / scale[:, None], "scale": scale}


def _exact_w4(s):
    w, ws, x = s["w"], s["ws"].double(), s["x"].double()
    n, groups = ws.shape
    group = 2 * w.shape[1] // groups
    y = torch.zeros(x.shape[0], n, dtype=torch.float64, device=DEV)
    for i in range(groups):
        b = w[:, i * group // 2:(i + 1) * group // 2].int()
        part = x[:, i * group:(i + 1) * group]
        y += (part[:, 0::2] @ ((b % 16) - 8).double().t() + part[:, 1::2] @ ((b // 16) - 8).double().t()) * ws[:, i]
    return y if s["xs"] is None else y * s["xs"].double()[:, None]


_EXACT = {"append": _exact_append, "attn": _exact_attn, "norm": _exact_norm, "w4": _exact_w4}


# ------------------------------------------------------------------ work

def work(case):
    """What a pass cannot do without: each input read and each output written once."""
    c = case
    if c["kind"] == "plan":
        ps = c["ps"]
        new = sum(_fresh(c)) / ps
        return {"bytes": 8 * c["B"] + 8 * new + 4 * (2 * c["B"] + 1) + 8 * sum(_fresh(c)), "flops": 0}
    if c["kind"] == "append":
        return {"bytes": c["N"] * (4 + 2 * 2 * 2 * c["hkv"] * c["d"]), "flops": 0}
    if c["kind"] == "attn":
        n = _attn_lengths(c)
        seen = sum(x - _hidden(c, x)[1] for x in n)
        rows = sum(-(-x // c["ps"]) for x in n)
        return {"bytes": seen * c["hkv"] * c["d"] * 4 + c["B"] * (c["hq"] * c["d"] * 4 + 12) + 4 * rows,
                "flops": 4 * seen * c["hq"] * c["d"]}
    if c["kind"] == "norm":
        e = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": c["T"] * (c["d"] * (4 * e + 1) + 4) + c["d"] * e, "flops": 8 * c["T"] * c["d"]}
    n, k, T = c["n"], c["k"], c["T"]
    return {"bytes": n * k // 2 + 2 * n * (k // c["group"]) + T * (k * (2 if c["x"] == "bf16" else 1) + 2 * n),
            "flops": 2 * T * n * k}
