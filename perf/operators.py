"""Cases of the paged 8-bit KV cache (Kv8Cache): the tables that place it, the append that fills it, the attention that reads it.

The cache holds a sequence's tokens in pages of 64.  A complete page is kept in e4m3 with one power-of-two scale per kv head for
its keys and one for its values: the smallest that brings the page's largest magnitude to at most 448.  A row reads the pages
before its own in 8 bits and its own page in bf16, as the rows came; `limit` says how many keys it sees (causal: its position
plus one).  Pages come from a pool through a block table; free pages are a stack, whose top goes to the first sequence that grows.

A case is one of four kinds of pass:
  tables   the tables of a pass: pages for the sequences that grow, and every new row's slot, sequence and position.
  append   K and V rows enter the cache (with the tables of their pass) and are read back as they stand in it.
  attend   attention of a pass's rows over a cache that holds them.
  step     one layer of a decoding pass: tables, append, attention.
Head shapes are those of the models this library is used with: 32 / 8 heads of 128 (4B and 8B), 32 / 4 of 128 (the 30B-A3B
mixture), 14 / 2 of 64 (the drafter), 4 / 2 of 32 (tiny).
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 64
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS = [(32, 8, 128), (32, 4, 128), (14, 2, 64), (4, 2, 32)]


def _case(name, kind, heads, batch, lo, hi, new_lo, new_hi, dtype="bf16", mask="causal"):
    """lo .. hi: tokens that the sequences hold before the pass; new_lo .. new_hi: rows of the pass per sequence."""
    c = {"kind": kind, "hq": heads[0], "hkv": heads[1], "hd": heads[2], "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo,
         "new_hi": new_hi, "dtype": dtype, "mask": mask}
    return dict({"name": name}, **c) if name else c


def listed():
    b8, a3b, drafter = HEADS[0], HEADS[1], HEADS[2]
    return [
        # a verify pass of a small batch asks for its slots: one short launch
        _case("tables_step_b16", "tables", HEADS[3], 16, 200, 4000, 32, 32),
        # a thousand requests of all lengths are admitted at once: the largest tables
        _case("tables_admit_b1000", "tables", HEADS[3], 1000, 0, 0, 1, 1024),
        # a verify pass's rows of one layer, sixteen sequences at odd positions
        _case("append_block_b16", "append", b8, 16, 300, 3000, 32, 32),
        # a whole prompt of one layer
        _case("append_prompt_4096", "append", b8, 1, 0, 0, 4096, 4096),
        # pieces of prompts that go on in the middle of a page, float32 rows, small heads
        _case("append_pieces_f32", "append", drafter, 7, 33, 1500, 1, 700, dtype="f32"),
        # one token of one sequence: the smallest attention
        _case("attend_token_b1", "attend", b8, 1, 4095, 4095, 1, 1),
        # one token each of sixteen long contexts: bound by the cache
        _case("attend_token_long_b16", "attend", b8, 16, 32767, 32767, 1, 1),
        # the benchmark's verify pass
        _case("attend_block_8b", "attend", b8, 1, 4095, 4095, 32, 32),
        # sixteen long contexts under a verify pass of 32 rows
        _case("attend_block_long_b16", "attend", b8, 16, 32736, 32736, 32, 32),
        # a prompt's causal attention
        _case("attend_prompt_4096", "attend", b8, 1, 0, 0, 4096, 4096),
        # a drafter's block, every row of which sees all of the block, float32, odd numbers of rows
        _case("attend_draft_f32_b7", "attend", drafter, 7, 500, 6000, 5, 31, dtype="f32", mask="block"),
        # one layer of a decoding pass of the mixture's heads
        _case("step_a3b_b8", "step", a3b, 8, 300, 3000, 17, 17),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["tables", "append", "attend", "attend", "attend", "step"])
    heads = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "tables":
        batch, new = spread(1, 1000), spread(1, 1024)
        hi = rng.choice([0, spread(1, 4096)])
        return _case(None, kind, HEADS[3], batch, hi // 4, hi, max(1, new // 4), new)
    prompt = rng.random() < 0.3
    batch = spread(1, 8) if prompt else spread(1, 16)
    if prompt:      # whole prompts, or pieces of them behind some tokens
        new = max(1, spread(40, 3000) // batch)
        hi = rng.choice([0, spread(1, 3000) // batch])
    else:           # decoding: one token, or a block
        new = rng.choice([1, rng.randint(1, 33)])
        hi = spread(16, 16000)
    mask = "block" if new <= 64 and rng.random() < 0.3 else "causal"
    return _case(None, kind, heads, batch, int(hi * rng.uniform(0.2, 1.0)), hi, max(1, int(new * rng.uniform(0.3, 1.0))), new, dtype, mask)


# ------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------
def _spread(lo, hi, batch):
    """Numbers spread evenly over lo .. hi, in no particular order."""
    return [lo + int((hi - lo + 1) * ((0.5 + 0.6180339887 * b) % 1.0)) for b in range(batch)]


def _lens(case):
    return _spread(case["lo"], case["hi"], case["batch"]), _spread(case["new_lo"], case["new_hi"], case["batch"])


def _data(case, seed):
    """K and V rows of all tokens [batch][padded length][kv heads][head_dim] (bf16, or float32 behind the start of the pass), and q
    of the pass's rows, packed.  Keys have channels of different size, as rotated keys of trained models do."""
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 17)
    start, new = _lens(case)
    total = max(s + n for s, n in zip(start, new))
    shape = (case["batch"], -(-total // PAGE) * PAGE, case["hkv"], case["hd"])
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    chan = torch.exp(0.7 * rnd(case["hkv"], case["hd"]))
    dt = DTYPES[case["dtype"]]
    k = torch.empty(shape, dtype=dt, device="cuda")
    v = torch.empty(shape, dtype=dt, device="cuda")
    for b in range(case["batch"]):
        k[b] = (rnd(*shape[1:]) * chan).to(dt)
        v[b] = rnd(*shape[1:]).to(dt)
    q = (1.5 * rnd(sum(new), case["hq"], case["hd"]) / (1 + chan.mean())).to(dt)
    return start, new, k, v, q


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(start, new):
    """Sequence and position of every row of a pass, the rows of a sequence one after the other."""
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
    cu = torch.cumsum(torch.tensor(new, device="cuda"), 0) - torch.tensor(new, device="cuda")
    at = torch.arange(sum(new), device="cuda") - cu[seq]
    return seq, torch.tensor(start, device="cuda")[seq] + at, at


def _quantised(x):
    """x [..., 64 tokens, heads, head_dim] in float32: the page as e4m3, and its scales [..., 1, heads, 1]."""
    amax = x.abs().amax(dim=(-3, -1), keepdim=True)
    m, e = torch.frexp(amax / 448)                     # amax / 448 = m 2^e, 0.5 <= m < 1: the scale is 2^e, or 2^(e-1) where m = 0.5
    e = torch.where(m == 0.5, e - 1, e)
    scale = torch.where(amax > 0, ((e + 127) << 23).view(torch.float32), torch.ones_like(m))      # 2^e by its bits
    return (x / scale).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    if case["kind"] == "tables":
        start, new = _lens(case)
        gen = torch.Generator().manual_seed(seed)      # which request has which length
        order = torch.randperm(len(start), generator=gen).tolist()
        start, new = [start[i] for i in order], [new[i] for i in order]
        k = v = q = None
    else:
        start, new, k, v, q = _data(case, seed)
    batch, end = case["batch"], [s + n for s, n in zip(start, new)]
    max_seq = -(-max(end) // PAGE) * PAGE
    s = {"case": case, "start": _int(start), "new": _int(new), "rows": sum(new), "max_new": max(new), "max_len": max(end), "q": q,
         "pages": sum(-(-e // PAGE) for e in end), "fresh": max(start) == 0, "none": _int([0] * batch), "limits": None,
         "max_seq": max_seq}
    seq, pos, at = _rows(start, new)
    if case["mask"] == "block":
        s["limits"] = _int(end)[seq]
    if k is not None:
        s["k"], s["v"] = k[seq, pos].contiguous(), v[seq, pos].contiguous()
    if own:
        from paper_2512_15176_amd import Kv8Cache
        step = max(PAGE, (1 << 16) // batch // PAGE * PAGE)      # the tokens before the pass enter in pieces, page by page of all sequences
        s["kv"] = kv = Kv8Cache(1, case["hq"], case["hkv"], case["hd"], batch, max_seq, n_pages=s["pages"],
                                max_rows=max(s["rows"], batch * step if max(start) else 1))
        for c0 in range(0, max(start), step):
            a, b = [min(x, c0) for x in start], [min(x, c0 + step) for x in start]
            n = [y - x for x, y in zip(a, b)]
            kv.reserve(_int(a), _int(n), sum(n), max(n), max(b))
            if k is not None:
                sq, ps, _ = _rows(a, n)
                kv.append(0, k[sq, ps], v[sq, ps])
        if case["kind"] == "attend":
            kv.reserve(s["start"], s["new"], s["rows"], s["max_new"], s["max_len"])
            kv.append(0, s["k"], s["v"])
    elif case["kind"] == "tables":
        # what the sequences hold before the pass: pages that came to them piece by piece, in the order of the requests
        held = [-(-x // PAGE) for x in start]
        table = torch.full((batch, max_seq // PAGE), -1, dtype=torch.int32)
        step, at_page, top = max(PAGE, (1 << 16) // batch // PAGE * PAGE), [0] * batch, 0
        for c0 in range(0, max(start), step):
            for b in range(batch):
                upto = -(-min(start[b], c0 + step) // PAGE)
                table[b, at_page[b]:upto] = torch.arange(top, top + upto - at_page[b], dtype=torch.int32)
                top += upto - at_page[b]
                at_page[b] = max(at_page[b], upto)
        s["table"], s["held"], s["top"] = table.cuda(), _int(held), top
    else:
        s.update(_plain_cache(case, start, new, k, v))
    return s


def _plain_cache(case, start, new, k, v):
    """The cache as a program without the operators holds it: e4m3 pages and scales, the pages of the pass in bf16."""
    batch, pages = k.shape[0], k.shape[1] // PAGE
    split = (batch, pages, PAGE, case["hkv"], case["hd"])
    k16, v16 = k.to(torch.bfloat16).view(split), v.to(torch.bfloat16).view(split)
    first = _int([x // PAGE for x in start])
    last = _int([(x + n - 1) // PAGE for x, n in zip(start, new)])
    width = int((last - first).max()) + 1
    index = (first[:, None] + torch.arange(width, device="cuda")).clamp(max=pages - 1).long()
    rows = torch.arange(batch, device="cuda")[:, None]
    s = {"k16": k16[rows, index], "v16": v16[rows, index], "first": first}
    if case["kind"] != "append":
        k8, v8 = torch.empty(split, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(split, dtype=torch.float8_e4m3fn, device="cuda")
        ks, vs = torch.empty(split[:2] + (1, case["hkv"], 1), device="cuda"), torch.empty(split[:2] + (1, case["hkv"], 1), device="cuda")
        for b in range(batch):
            k8[b], ks[b] = _quantised(k16[b].float())
            v8[b], vs[b] = _quantised(v16[b].float())
        s.update({"k8": k8, "v8": v8, "ks": ks, "vs": vs})
    return s


# ------------------------------------------------------------------------------------------------------------------
# the passes
# ------------------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        kv = s["kv"]
        if kind != "attend":
            if s["fresh"]:      # the requests before these ones have ended
                kv.reserve(s["none"], s["none"], 0, 0, 0)
            slots = kv.reserve(s["start"], s["new"], s["rows"], s["max_new"], s["max_len"])
        if kind == "tables":
            return {"table": kv.block_table, "slots": slots, "seq": kv.row_seq[:s["rows"]], "pos": kv.row_pos[:s["rows"]]}
        if kind != "attend":
            kv.append(0, s["k"], s["v"])
        if kind == "append":
            k, v = kv.read(0, kv.row_seq[:s["rows"]], kv.row_pos[:s["rows"]])
            return {"k": k, "v": v}
        return {"out": kv.attend(0, s["q"], limits=s["limits"])}
    if kind == "tables":
        return _plain_tables(s)
    if kind == "append":
        return _plain_append(s)
    if kind == "step":
        s = _plain_enter(s)
    return {"out": _plain_attend(s)}


def _plain_rows(s):
    new = s["new"].long()
    cu = torch.cumsum(new, 0) - new
    seq = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new, output_size=s["rows"])
    at = torch.arange(s["rows"], device="cuda") - cu[seq]
    return seq, s["start"].long()[seq] + at, at


def _plain_tables(s):
    seq, pos, _ = _plain_rows(s)
    need = (s["start"] + s["new"] + PAGE - 1) // PAGE
    grow = need - s["held"]                                       # no sequence of these passes gives pages back
    base = s["top"] + torch.cumsum(grow, 0, dtype=torch.int32) - grow      # the pool's pages are handed out in order
    col = torch.arange(s["table"].shape[1], dtype=torch.int32, device="cuda")[None]
    fresh = (col >= s["held"][:, None]) & (col < need[:, None])
    table = torch.where(fresh, base[:, None] + col - s["held"][:, None], s["table"])
    slots = table[seq, pos // PAGE] * PAGE + (pos % PAGE).int()
    return {"table": table, "slots": slots, "seq": seq.int(), "pos": pos.int()}


def _plain_entered(s):
    """The pages of the pass with its rows in them, bf16."""
    seq, pos, _ = _plain_rows(s)
    at = (seq, pos // PAGE - s["first"].long()[seq], pos % PAGE)
    k16, v16 = s["k16"].clone(), s["v16"].clone()
    k16[at], v16[at] = s["k"].to(torch.bfloat16), s["v"].to(torch.bfloat16)
    return k16, v16, at


def _plain_append(s):
    k16, v16, at = _plain_entered(s)
    whole = (s["first"].long()[at[0]] + at[1] + 1) * PAGE <= (s["start"] + s["new"])[at[0]]   # the row's page is complete
    k8, ks = _quantised(k16.float())
    v8, vs = _quantised(v16.float())
    pick = lambda x8, sc, x16: torch.where(whole[:, None, None], (x8.float() * sc)[at].to(torch.bfloat16), x16[at])   # noqa: E731
    return {"k": pick(k8, ks, k16), "v": pick(v8, vs, v16)}


def _plain_enter(s):
    """A pass's rows enter the plain cache: its pages in bf16, and in 8 bits where they are read so."""
    k16, v16, _ = _plain_entered(s)
    pages = s["first"].long()[:, None] + torch.arange(k16.shape[1], device="cuda")
    index = (torch.arange(k16.shape[0], device="cuda")[:, None], pages.clamp(max=s["k8"].shape[1] - 1))
    s = dict(s, k16=k16, v16=v16, k8=s["k8"].clone(), v8=s["v8"].clone(), ks=s["ks"].clone(), vs=s["vs"].clone())
    (k8, ks), (v8, vs) = _quantised(k16.float()), _quantised(v16.float())
    s["k8"].view(torch.uint8)[index], s["v8"].view(torch.uint8)[index] = k8.view(torch.uint8), v8.view(torch.uint8)
    s["ks"][index], s["vs"][index] = ks, vs
    return s


def _plain_attend(s):
    c = s["case"]
    batch, hkv, hd, group, n = c["batch"], c["hkv"], c["hd"], c["hq"] // c["hkv"], s["max_new"]
    seq, pos, at = _plain_rows(s)
    limit = pos + 1 if s["limits"] is None else s["limits"].long()
    page = (limit - 1) // PAGE
    fill = lambda x: torch.zeros((batch, n) + x.shape[1:], dtype=x.dtype, device="cuda").index_put((seq, at), x)   # noqa: E731
    q = fill(s["q"].float() / math.sqrt(hd)).view(batch, n, hkv, group, hd)
    own_page, limit_of = fill(page - s["first"].long()[seq]), fill(limit)
    first_own = fill(page) * PAGE                                # keys before it are read in 8 bits
    k8 = (s["k8"].float() * s["ks"]).view(batch, -1, hkv, hd).permute(0, 2, 3, 1).contiguous()
    s8 = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(batch, hkv, n * group, hd), k8).view(batch, hkv, n, group, -1)
    key = torch.arange(s8.shape[-1], device="cuda")
    s8 = s8.masked_fill_((key >= first_own[..., None])[:, None, :, None], -math.inf)
    rows = torch.arange(batch, device="cuda")[:, None]
    k16 = s["k16"][rows, own_page].float().permute(0, 1, 3, 4, 2).contiguous()         # [batch][n][kv head][hd][64]
    s16 = torch.matmul(q, k16).permute(0, 2, 1, 3, 4)                                   # [batch][kv head][n][group][64]
    key16 = first_own[..., None] + torch.arange(PAGE, device="cuda")
    s16 = s16.masked_fill((key16 >= limit_of[..., None])[:, None, :, None], -math.inf)
    m = torch.maximum(s8.amax(-1), s16.amax(-1))[..., None]
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    p8, p16 = torch.exp(s8 - m), torch.exp(s16 - m)
    total = p8.sum(-1) + p16.sum(-1)
    v8 = (s["v8"].float() * s["vs"]).view(batch, -1, hkv, hd).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p8.view(batch, hkv, n * group, -1), v8).view(batch, hkv, n, group, hd)
    v16 = s["v16"][rows, own_page].float().permute(0, 3, 1, 2, 4).contiguous()          # [batch][kv head][n][64][hd]
    o = (o + torch.matmul(p16, v16)) / total.clamp(min=1e-30)[..., None]
    return o.permute(0, 2, 1, 3, 4).reshape(batch, n, c["hq"], hd)[seq, at].to(s["q"].dtype)


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    start, new = _lens(case)
    rows, esz = sum(new), 2 if case["dtype"] == "bf16" else 4
    fresh = [-(-(a + n) // PAGE) - -(-a // PAGE) for a, n in zip(start, new)]
    tables = 16 * len(start) + 12 * rows + 4 * sum(fresh)
    if case["kind"] == "tables":
        return {"bytes": tables, "flops": 0}
    row = 2 * case["hkv"] * case["hd"]                               # elements of K and V of a token
    entered = rows * row * esz                                       # the rows are read
    for a, n in zip(start, new):
        whole, before = (a + n) // PAGE - a // PAGE, a % PAGE
        entered += whole * PAGE * row + (before * row * 2 if whole else 0)           # complete pages in 8 bits, their older rows read
        entered += ((a + n) % PAGE if whole else n) * row * 2                        # rows of the open page
    if case["kind"] == "append":
        return {"bytes": tables + entered + rows * row * 2 + rows * row, "flops": rows * row * 4}
    read = flops = 0
    for a, n in zip(start, new):
        last = a + n
        read += (last - 1) // PAGE * PAGE * row                                      # pages before the last row's own, in 8 bits
        read += (last - a // PAGE * PAGE) * row * 2                                  # the pages of the pass's own rows
        seen = n * last if case["mask"] == "block" else n * a + n * (n + 1) // 2
        flops += 4 * case["hd"] * case["hq"] * seen
    io = 2 * rows * case["hq"] * case["hd"] * esz
    return {"bytes": read + io + (tables + entered if case["kind"] == "step" else 0), "flops": flops}


# ------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, sequence by sequence
# ------------------------------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e in float64, exactly."""
    return ((e + 1023) << 52).view(torch.float64)


def _exponent(x):
    """The e with 2^e <= x < 2^(e+1), of normal float64 numbers."""
    return (x.view(torch.int64) >> 52) - 1023


def _page64(x):
    """A complete page [64][heads][head_dim] of bf16 rows as the values that its 8 bits stand for, float64."""
    out = x.double()
    top = out.abs().amax(dim=2).amax(dim=0).clamp(min=2.0 ** -80)
    e = _exponent(top) - 8
    s = _two_to(torch.where(top > 448 * _two_to(e), e + 1, e))[None, :, None]
    y = out / s
    # nearest e4m3, ties to even: a step is 2^-3 of the value's power of two, at least 2^-9
    step = _two_to(_exponent(y.abs().clamp(min=2.0 ** -6)) - 3)
    return torch.round(y / step) * step * s


def exact(case, seed):
    if case["kind"] == "tables":
        return None
    start, new, k, v, q = _data(case, seed)
    outs, ks, vs, r = [], [], [], 0
    hkv, hd, group = case["hkv"], case["hd"], case["hq"] // case["hkv"]
    for b, (a, n) in enumerate(zip(start, new)):
        end = a + n
        kb, vb = k[b, :end].to(torch.bfloat16), v[b, :end].to(torch.bfloat16)
        cut = end // PAGE * PAGE
        quant = lambda x: torch.cat([_page64(p) for p in x[:cut].split(PAGE)] + [x[cut:].double()]) if cut else x.double()   # noqa: E731
        k8, v8 = quant(kb), quant(vb)
        if case["kind"] == "append":
            ks.append(k8[a:])
            vs.append(v8[a:])
            continue
        qb = q[r:r + n].double().view(n, hkv, group, hd) / math.sqrt(hd)
        r += n
        limit = torch.full((n,), end, device="cuda") if case["mask"] == "block" else torch.arange(a, end, device="cuda") + 1
        out = torch.empty(n, hkv, group, hd, dtype=torch.float64, device="cuda")
        edges = sorted({0, n} | {i for i in range(1, n) if (int(limit[0]) - 1 + i) % PAGE == 0 and case["mask"] == "causal"})
        for i0, i1 in zip(edges, edges[1:]):                         # the rows of one page see the same 8-bit keys
            own_page = (int(limit[i1 - 1]) - 1) // PAGE * PAGE
            top = int(limit[i1 - 1])
            kk = torch.cat([k8[:own_page], kb[own_page:top].double()]).permute(1, 2, 0)
            vv = torch.cat([v8[:own_page], vb[own_page:top].double()]).permute(1, 0, 2)
            sc = torch.matmul(qb[i0:i1].permute(1, 0, 2, 3).reshape(hkv, -1, hd), kk.contiguous()).view(hkv, i1 - i0, group, top)
            hidden = torch.arange(top, device="cuda")[None] >= limit[i0:i1, None]
            p = torch.softmax(sc.masked_fill(hidden[None, :, None], -math.inf), -1)
            out[i0:i1] = torch.matmul(p.view(hkv, -1, top), vv.contiguous()).view(hkv, i1 - i0, group, hd).permute(1, 0, 2, 3)
        outs.append(out.view(n, case["hq"], hd))
    if case["kind"] == "append":
        return {"k": torch.cat(ks), "v": torch.cat(vs)}
    return {"out": torch.cat(outs)}
