"""Operators of serving on a key-value cache held in 4 bits, and of scoring what a
model answers: what is measured.

Four operators, in the order in which a server calls them:

  store   a chunk's new key and value rows quantised into the pages of a cache in
          4 bits (append), and the rows that the chunk's attention needs read
          back in bf16 (read): two operators, run together as a chunk runs them
  attn    attention of one new token per request over its 4-bit pages, the hidden
          (visual) block of a request left out
  logp    log probabilities of given tokens from the logits, with each row's
          entropy and its most probable alternatives

A pool holds [num_pages, Hkv, page_size / 8, bytes] uint8: eight rows of a KV
head as the codes of their keys [8, D / 2], the parameters of their keys
[8, D / group, 2] bf16 (step, low), then the same two for their values. A code q
of a group stands for low + step q, q in 0..15, with low = the group's least
value and step = (its largest - its least) / 15 rounded to bf16. Order inside a
row of codes: the 32-bit word c (D / 32) + i of keys holds features
32 i + 8 c .. + 7, the 16-bit word r (D / 32) + i of values features
32 i + 4 r .. + 3, the lowest feature in the lowest four bits.

Where `own` is false, run() computes the plain form in elementary torch
operations in 32 bits. Layer shapes are the repository's own (32 query heads on
4 KV heads of 128, the 2049 rows of the text-only cache, 1552 rows, 16384 rows,
a vocabulary of 32001) or generic.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
SCRATCH = 64 << 20  # bytes of workspace that a serving program keeps for the attention


def listed():
    return [
        # One layer's new rows of a decode batch of odd size, and the same rows read.
        {"name": "store_decode_N23", "kind": "store", "N": 23, "C": 23, "hkv": 4, "d": 128, "group": 64, "ps": 16},
        # The last chunk of a long prompt: 1552 rows come in, its attention reads all 16384.
        {"name": "store_chunk_N1552", "kind": "store", "N": 1552, "C": 16384, "hkv": 4, "d": 128, "group": 64, "ps": 64},
        # A long prompt in one piece, on small heads with finer groups.
        {"name": "store_prompt_N16381", "kind": "store", "N": 16381, "C": 16381, "hkv": 8, "d": 64, "group": 32, "ps": 32},
        # One request over the text-only cache: the latency of a decode step.
        {"name": "attn_B1_C2049", "kind": "attn", "B": 1, "lo": 2049, "hi": 2049, "hide": 0.0, "hq": 32, "hkv": 4,
         "d": 128, "group": 64, "ps": 16, "empty": 0},
        # A full batch of long multimodal requests after the exit, their visual
        # blocks hidden: the largest call.
        {"name": "attn_B96_ragged", "kind": "attn", "B": 96, "lo": 2000, "hi": 16385, "hide": 0.6, "hq": 32, "hkv": 4,
         "d": 128, "group": 64, "ps": 64, "empty": 0},
        # Many short chats on a small model: heads of 64, a KV head for every
        # query head, and two slots of the batch without a request.
        {"name": "attn_B97_D64", "kind": "attn", "B": 97, "lo": 5, "hi": 1553, "hide": 0.0, "hq": 16, "hkv": 16,
         "d": 64, "group": 32, "ps": 32, "empty": 2},
        # Few KV heads for many query heads, one group per row, small pages.
        {"name": "attn_B24_G16", "kind": "attn", "B": 24, "lo": 100, "hi": 4001, "hide": 0.0, "hq": 32, "hkv": 2,
         "d": 128, "group": 128, "ps": 8, "empty": 0},
        # The next token of one request, with five alternatives: latency.
        {"name": "logp_T1_V32001", "kind": "logp", "T": 1, "V": 32001, "n": 5, "dtype": "bf16", "pad": 0, "masked": 0.0},
        # A decode batch over a large vocabulary of odd size in fp32, a third of
        # it ruled out by a grammar.
        {"name": "logp_T24_V151001", "kind": "logp", "T": 24, "V": 151001, "n": 20, "dtype": "f32", "pad": 0,
         "masked": 0.33},
        # A prompt scored token by token (its last rows are padding).
        {"name": "logp_T1552_V32001", "kind": "logp", "T": 1552, "V": 32001, "n": 0, "dtype": "bf16", "pad": 7,
         "masked": 0.0},
        # The longest prompt scored with alternatives: the largest call.
        {"name": "logp_T16384_V32001", "kind": "logp", "T": 16384, "V": 32001, "n": 5, "dtype": "bf16", "pad": 0,
         "masked": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "store", "attn", "attn", "attn", "logp", "logp"])
    d = rng.choice([64, 128, 128])
    group = rng.choice([32, 64] if d == 64 else [32, 64, 128])
    ps = rng.choice([8, 16, 32, 64, 128])
    if kind == "store":
        hkv = rng.choice([1, 2, 4, 8])
        C = _log(rng, 1, 16384 * 512 // max(512, hkv * d))
        N = rng.choice([C, max(1, C // 10), min(C, _log(rng, 1, 2000))])
        return {"kind": "store", "N": N, "C": C, "hkv": hkv, "d": d, "group": group, "ps": ps}
    if kind == "attn":
        hkv, per = rng.choice([(1, 8), (4, 8), (4, 8), (8, 4), (2, 16), (8, 1), (4, 6), (5, 5)])
        # keys in all, by the bytes that the largest listed case reads
        most = 250_000 * 512 // (hkv * d)
        hi = _log(rng, 3, 40_000)
        B = min(_log(rng, 1, 200), max(1, most // hi))
        lo = rng.choice([1, max(1, hi // 8), hi])
        return {"kind": "attn", "B": B, "lo": lo, "hi": hi, "hide": rng.choice([0.0, 0.0, 0.5, 0.9]), "hq": hkv * per,
                "hkv": hkv, "d": d, "group": group, "ps": ps, "empty": rng.choice([0, 0, 1]) if B > 1 else 0}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    V = _log(rng, 2, 260_000)
    T = min(_log(rng, 1, 16384), max(1, 16384 * 32001 // V // (2 if dtype == "f32" else 1)))
    return {"kind": "logp", "T": T, "V": V, "n": min(V, rng.choice([0, 1, 5, 20, 32])), "dtype": dtype,
            "pad": rng.choice([0, 0, 1]) if T > 1 else 0, "masked": rng.choice([0.0, 0.0, 0.5])}


# ------------------------------------------------------------------ inputs

def _lengths(c):
    """The requests' lengths: spread evenly over the logarithm of [lo, hi]."""
    lo, hi, B = c["lo"], c["hi"], c["B"]
    a, b = math.log(lo + 1.0), math.log(hi + 1.0)
    n = [int(round(math.exp(a + (b - a) * (i + 1) / B))) - 1 for i in range(B)]
    return [0] * c["empty"] + n[c["empty"]:]


def _hidden(c, n):
    """(begin, count) of the hidden block of a request of n rows."""
    return (min(16, n // 8), int(n * c["hide"])) if c["hide"] else (0, 0)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _rows(g, n, hkv, d):
    """n key or value rows: some features of a head run larger, and off centre, as keys' do."""
    x = torch.randn(n, hkv, d, generator=g, device=DEV)
    x[..., 3::17] = x[..., 3::17] * 4 + 2
    return x.to(torch.bfloat16)


def _pool(g, pages, c):
    """A pool whose rows have all been stored."""
    tiles = pages * c["ps"] // 8
    part = max(1, (1 << 26) // (c["hkv"] * c["d"] * 8))
    out = torch.empty(tiles, c["hkv"], 8 * (c["d"] + 8 * (c["d"] // c["group"])), dtype=torch.uint8, device=DEV)
    for i in range(0, tiles, part):
        n = min(part, tiles - i)
        rows = [_rows(g, 8 * n, c["hkv"], c["d"]) for _ in range(2)]
        out[i:i + n] = torch.cat([x.unflatten(0, (n, 8)).transpose(1, 2).flatten(2) for kv in range(2)
                                  for x in _pack(*_quantise(rows[kv], c["group"]), kv)], 2)
    return out.view(pages, c["ps"] // 8, c["hkv"], -1).transpose(1, 2).contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 17)
    return _PREPARE[case["kind"]](case, g)


def _prepare_store(c, g):
    N, C, hkv, d, ps = c["N"], c["C"], c["hkv"], c["d"], c["ps"]
    # the rows as a fused projection leaves them: keys and values inside wider rows
    qkv = torch.cat([_rows(g, N, 2 * hkv, d), _rows(g, N, hkv, d), _rows(g, N, hkv, d)], 1)
    if N == C and N <= 200:  # a decode batch: rows anywhere
        P = 2 * N // ps + 3
        slots = torch.randperm(P * ps, generator=g, device=DEV)[:C]
    else:  # one request, its pages in any order
        P = -(-C // ps) + 3
        j = torch.arange(C, device=DEV)
        slots = torch.randperm(P, generator=g, device=DEV)[j // ps] * ps + j % ps
    slots = slots.to(torch.int32)
    e = lambda: torch.empty(C, hkv, d, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    return {"case": c, "k": qkv[:, 2 * hkv:3 * hkv], "v": qkv[:, 3 * hkv:], "slots": slots, "new": slots[C - N:],
            "pages": _pool(g, P, c), "k_out": e(), "v_out": e()}


def _prepare_attn(c, g):
    B, ps, hq, hkv, d = c["B"], c["ps"], c["hq"], c["hkv"], c["d"]
    n = _lengths(c)
    order = torch.randperm(B, generator=g, device=DEV)
    hid = [_hidden(c, x) for x in n]
    lens, hb, hc = _i32(n)[order], _i32([h[0] for h in hid])[order], _i32([h[1] for h in hid])[order]
    width = max(1, -(-max(n) // ps))
    used = -(-lens // ps)
    P = sum(-(-x // ps) for x in n) + 8
    pages = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
    cols = torch.arange(width, device=DEV)[None]
    start = (torch.cumsum(used, 0) - used)[:, None]
    # pages that lie wholly inside a hidden block have been given back
    gone = (cols * ps >= hb[:, None]) & ((cols + 1) * ps <= (hb + hc)[:, None])
    table = torch.where((cols < used[:, None]) & ~gone, pages[(start + cols).clamp(max=P - 1)], -1).to(torch.int32)
    q = torch.randn(B, hq + 2 * hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    return {"case": c, "q": q[:, :hq], "pages": _pool(g, P, c), "table": table, "lens": lens,
            "hb": hb if c["hide"] else None, "hc": hc if c["hide"] else None,
            "out": torch.empty(B, hq, d, dtype=torch.bfloat16, device=DEV),
            "ws": torch.empty(SCRATCH, dtype=torch.uint8, device=DEV)}


def _prepare_logp(c, g):
    T, V, n = c["T"], c["V"], c["n"]
    x = torch.empty(T, V, dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32, device=DEV)
    x.normal_(0, 2.5, generator=g)
    # some rows are all but certain of one token
    sure = torch.arange(0, T, 3, device=DEV)
    x[sure, torch.randint(0, V, (len(sure),), generator=g, device=DEV)] = 17.0
    if c["masked"]:
        x[:, torch.rand(V, generator=g, device=DEV) < c["masked"]] = -math.inf
        x[:, 0] = 0.25
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV).to(torch.int32)
    if c["pad"]:
        tokens[T - min(c["pad"], T - 1):] = -1
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=DEV)  # noqa: E731
    return {"case": c, "x": x, "tokens": tokens, "logprob": z(T), "entropy": z(T), "top_id": z(T, n, t=torch.int32),
            "top_logprob": z(T, n)}


_PREPARE = {"store": _prepare_store, "attn": _prepare_attn, "logp": _prepare_logp}


# ------------------------------------------------------------------ the calls

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


def _own_store(s):
    import paper_2609_38823_gb300 as dm

    dm.decomoe_paged_append_q4(s["k"], s["v"], s["new"], s["pages"])
    dm.decomoe_paged_read_q4(s["slots"], s["pages"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attn(s):
    import paper_2609_38823_gb300 as dm

    dm.decomoe_paged_attention_q4(s["q"], s["pages"], s["table"], s["lens"], s["out"], s["ws"], hide_begin=s["hb"],
                                  hide_count=s["hc"])
    return s["out"]


def _own_logp(s):
    import paper_2609_38823_gb300 as dm

    n = s["case"]["n"]
    dm.decomoe_token_logprobs(s["x"], s["tokens"], s["logprob"], s["entropy"], s["top_id"] if n else None,
                              s["top_logprob"] if n else None)
    return {k: s[k] for k in ("logprob", "entropy") + (("top_id", "top_logprob") if n else ())}


_OWN = {"store": _own_store, "attn": _own_attn, "logp": _own_logp}


# ------------------------------------------------------------------ plain forms

def _quantise(x, group):
    """Codes [..., d] and parameters [..., d / group, 2] bf16 of rows. The places of values
    between two codes are computed in 64 bits."""
    x = x.double().unflatten(-1, (-1, group))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    step = ((hi - lo) / 15).to(torch.bfloat16).double()
    q = torch.where(step > 0, torch.round((x - lo) / torch.where(step > 0, step, 1)), 0).clamp(0, 15)
    return q.flatten(-2).to(torch.uint8), torch.cat([step, lo], -1).to(torch.bfloat16)


# places of the features in a row's bytes: [c, i, feature] of keys, [r, i, feature] of values
_LANES, _RUN = (4, 8), (8, 4)


def _pack(codes, params, kv):
    """(bytes of the codes, bytes of the parameters) of rows."""
    c = codes.unflatten(-1, (-1, _LANES[kv], _RUN[kv])).transpose(-3, -2).flatten(-3)
    return c[..., 0::2] | c[..., 1::2] << 4, params.flatten(-2).contiguous().view(torch.uint8)


def _tile_parts(tiles, d, group):
    """[(codes [..., 8, d / 2], parameters [..., 8, d / group, 2] bf16) of keys and of values],
    views of the bytes of tiles."""
    sizes = [4 * d, 32 * (d // group)] * 2
    k, kp, v, vp = torch.split(tiles, sizes, -1)
    part = lambda c, p: (c.unflatten(-1, (8, -1)), p.unflatten(-1, (8, -1)))  # noqa: E731
    return [part(k, kp), part(v, vp)]


def _values(codes, params, kv, d, group):
    """The fp32 values of rows from their bytes."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    q = q.unflatten(-1, (_LANES[kv], d // 32, _RUN[kv])).transpose(-3, -2).flatten(-3)
    p = params.contiguous().view(torch.bfloat16).float().unflatten(-1, (-1, 2))
    return (p[..., 1:] + p[..., :1] * q.float().unflatten(-1, (-1, group))).flatten(-2)


def _plain_store(s):
    c = s["case"]
    d, group, tiles_of = c["d"], c["group"], s["pages"].shape[2]
    new, every = s["new"].long(), s["slots"].long()
    parts = _tile_parts(s["pages"], d, group)
    out = []
    for kv, x in enumerate((s["k"], s["v"])):
        at = (new // (8 * tiles_of), slice(None), new // 8 % tiles_of, new % 8)
        for dst, src in zip(parts[kv], _pack(*_quantise(x, group), kv)):
            dst[at] = src
        at = (every // (8 * tiles_of), slice(None), every // 8 % tiles_of, every % 8)
        out.append(_values(*(p[at] for p in parts[kv]), kv, d, group).to(torch.bfloat16))
    return {"k": out[0], "v": out[1]}


def _plain_attn(s):
    q, table, lens, c = s["q"], s["table"], s["lens"], s["case"]
    B, hq, d = q.shape
    hkv = c["hkv"]
    tiles = s["pages"][table.clamp(min=0).long()]  # [B, pages, hkv, tiles, bytes]
    tiles = tiles.transpose(2, 3).flatten(1, 2)
    k, v = (_values(*p, kv, d, c["group"]).transpose(2, 3).flatten(1, 2)
            for kv, p in enumerate(_tile_parts(tiles, d, c["group"])))  # [B, keys, hkv, d]
    j = torch.arange(k.shape[1], device=DEV)[None]
    see = j < lens[:, None]
    if s["hb"] is not None:
        see &= (j < s["hb"][:, None]) | (j >= (s["hb"] + s["hc"])[:, None])
    x = torch.einsum("bghd,bkgd->bghk", q.reshape(B, hkv, hq // hkv, d).float(), k) / math.sqrt(d)
    x = torch.where(see[:, None, None], x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0, m))
    o = torch.einsum("bghk,bkgd->bghd", p, v)
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, o / torch.where(total > 0, total, 1), 0)
    return o.reshape(B, hq, d).to(torch.bfloat16)


def _plain_logp(s):
    n, keep = s["case"]["n"], s["tokens"] >= 0
    x = s["x"].float()
    m = x.amax(-1, keepdim=True)
    y = x - m
    e = torch.exp(y)
    total = e.sum(-1)
    lse = torch.log(total)
    entropy = lse - torch.where(e > 0, e * y, 0).sum(-1) / total
    logprob = y.gather(1, s["tokens"].clamp(min=0).long()[:, None])[:, 0] - lse
    out = {"logprob": torch.where(keep, logprob, s["logprob"]), "entropy": torch.where(keep, entropy, s["entropy"])}
    if n:
        del e
        best, at = torch.sort(y, dim=-1, descending=True, stable=True)
        out["top_id"] = torch.where(keep[:, None], at[:, :n].to(torch.int32), s["top_id"])
        out["top_logprob"] = torch.where(keep[:, None], best[:, :n] - lse[:, None], s["top_logprob"])
    return out


_PLAIN = {"store": _plain_store, "attn": _plain_attn, "logp": _plain_logp}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """run()'s outputs from the definitions in 64 bits, one request, head or block
    of rows at a time; None for whole-number outputs."""
    return _EXACT[case["kind"]](prepare(case, seed))


def _exact_cached(s, slots, head):
    """(keys, values) [rows, d] in 64 bits of one head's rows of the cache, feature by feature
    from the layout of a tile."""
    c = s["case"]
    d, group, ps = c["d"], c["group"], c["ps"]
    tile = s["pages"][slots // ps, head, slots % ps // 8]
    row, f = (slots % 8)[:, None], torch.arange(d, device=DEV)[None]
    halves = tile.shape[1] // 2
    out = []
    for base, step, run in ((0, 4, 8), (halves, 8, 4)):
        i, rest = f // 32, f % 32
        nibble = (rest // run * (d // 32) + i) * run + rest % run
        byte = tile.gather(1, base + row * (d // 2) + nibble // 2)
        code = torch.where(nibble % 2 == 1, byte // 16, byte % 16).double()
        at = base + 4 * d + (row * (d // group) + f // group) * 4
        bf = lambda k: ((tile.gather(1, at + k).int() + 256 * tile.gather(1, at + k + 1).int()) << 16).view(torch.float32)  # noqa: E731
        out.append(bf(2).double() + bf(0).double() * code)
    return out


def _exact_store(s):
    c = s["case"]
    out = {}
    for i, (name, x) in enumerate((("k", s["k"]), ("v", s["v"]))):
        old = torch.stack([_exact_cached(s, s["slots"][:c["C"] - c["N"]].long(), h)[i] for h in range(c["hkv"])], 1)
        y = x.double().reshape(c["N"], c["hkv"], -1, c["group"])
        low = torch.min(y, -1, keepdim=True)[0]
        step = ((torch.max(y, -1, keepdim=True)[0] - low) / 15).float().bfloat16().double()
        code = torch.nan_to_num((y - low) / step).round().clamp(0, 15)
        out[name] = torch.cat([old, (low + code * step).reshape(x.shape)])
    return out


def _exact_attn(s):
    B, hq, d = s["q"].shape
    hkv, ps = s["case"]["hkv"], s["case"]["ps"]
    out = torch.zeros(B, hq, d, dtype=torch.float64, device=DEV)
    lens = s["lens"].tolist()
    hide = [(0, 0)] * B if s["hb"] is None else list(zip(s["hb"].tolist(), s["hc"].tolist()))
    for b in range(B):
        h0, h1 = hide[b][0], hide[b][0] + hide[b][1]
        j = torch.tensor([i for i in range(lens[b]) if not h0 <= i < h1], dtype=torch.long, device=DEV)
        if not len(j):
            continue
        slots = s["table"][b].long()[j // ps] * ps + j % ps
        for h in range(hkv):
            k, v = _exact_cached(s, slots, h)
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            x = s["q"][b, heads].double() @ k.t() * d ** -0.5
            out[b, heads] = torch.softmax(x, -1) @ v
    return out


def _exact_logp(s):
    T, n = s["case"]["T"], s["case"]["n"]
    out = {"logprob": s["logprob"].double(), "entropy": s["entropy"].double()}
    if n:
        out |= {"top_id": None, "top_logprob": s["top_logprob"].double()}
    rows = max(1, (1 << 27) // s["case"]["V"])
    for i in range(0, T, rows):
        at = torch.nonzero(s["tokens"][i:i + rows] >= 0)[:, 0] + i
        lp = torch.log_softmax(s["x"][at].double(), -1)
        out["logprob"][at] = lp[torch.arange(len(at), device=DEV), s["tokens"][at].long()]
        out["entropy"][at] = torch.special.entr(torch.exp(lp)).sum(-1)
        if n:
            out["top_logprob"][at] = torch.topk(lp, n, -1).values
    return out


_EXACT = {"store": _exact_store, "attn": _exact_attn, "logp": _exact_logp}


# ------------------------------------------------------------------ work

def work(case):
    """What a pass cannot do without: each input read and each output written once."""
    c = case
    if c["kind"] == "logp":
        e = 2 if c["dtype"] == "bf16" else 4
        rows = c["T"] - min(c["pad"], c["T"] - 1)
        return {"bytes": rows * (c["V"] * e + 12 + 8 * c["n"]), "flops": 5 * rows * c["V"]}
    held = c["hkv"] * (c["d"] + 8 * (c["d"] // c["group"]))  # bytes of a cached row
    if c["kind"] == "store":
        full = 4 * c["hkv"] * c["d"]
        return {"bytes": (c["N"] + c["C"]) * (full + held + 4), "flops": 2 * c["hkv"] * c["d"] * (8 * c["N"] + 2 * c["C"])}
    n = _lengths(c)
    seen = sum(x - _hidden(c, x)[1] for x in n)
    rows = sum(-(-x // c["ps"]) for x in n)
    return {"bytes": seen * held + c["B"] * (c["hq"] * c["d"] * 4 + 12) + 4 * rows, "flops": 4 * seen * c["hq"] * c["d"]}
