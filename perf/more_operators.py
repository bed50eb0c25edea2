"""A quantised cache, its decode and blocks chosen by a cheap score: their calls, inputs, plain forms and 64-bit results.

A case is a dict of plain values.  `op` names the entry points:

  write   CacheQuantizer.write, .read   each sequence's last `new` tokens into a cache of `bits` bits, with the bounds of
                                        its blocks of `block` rows, and the values that were stored
  read    CacheQuantizer.read           rows of such a cache back in bf16
  decode  QuantizedDecoder(...)         one token per sequence over all of it, with capped scores and a distance bias
  select  BlockSelector(...)            the `budget` blocks of each KV head with the best bounds for the token
  blocks  BlockSelector, QuantizedDecoder  one token per sequence over the blocks chosen for it

`page` > 0 keeps the cache in pages of so many tokens, else every sequence has a span with room for more tokens.
Lists of numbers are comma-separated texts.

The cache: 128 values are four groups of 32 with a power of two each (a byte, 127 for 1); 8 bits are e4m3, 4 bits e2m1
with the first of two values in the lower half of the byte.  The power is the least that holds the group's largest value.
"""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128
DEV = "cuda"
SPARE = 37  # rows of a span behind its sequence
own = False


# ------------------------------------------------------------------------------------------ the cases
def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _text(values):
    return ",".join(str(int(x)) for x in values)


def _case(name, op, lens, hq, hkv, bits, page=0, block=0, **kw):
    return dict(name=name, op=op, lens=_text(lens), hq=hq, hkv=hkv, bits=bits, page=page, block=block, **kw)


def _write(name, lens, new, hkv, bits, page=0, block=0):
    return _case(name, "write", lens, hkv, hkv, bits, page, block, new=_text(new))


def _read(name, lens, new, hkv, bits, page=0):
    return _case(name, "read", lens, hkv, hkv, bits, page, new=_text(new))


def _decode(name, lens, hq, hkv, bits, page=0, cap=0.0, alibi=False):
    return _case(name, "decode", lens, hq, hkv, bits, page, cap=float(cap), alibi=alibi)


def _chosen(name, op, lens, hq, hkv, bits, block, budget, page=0, first=1, last=2):
    return _case(name, op, lens, hq, hkv, bits, page, block, budget=budget, first=first, last=last, cap=0.0, alibi=False)


def listed():
    chats = [(137 * i * i + 61 * i) % 1900 + 300 for i in range(32)]
    return [
        # a decode step of 32 conversations: one token each, bounds of the block it falls into
        _write("write_step_32", chats, [1] * 32, 8, 8, block=64),
        # a batch of prompts into pages at four bits
        _write("write_prompts_paged", [20000, 8192, 5001], [20000, 8192, 5001], 8, 4, page=64, block=32),
        # a long prompt's cache in bf16 again, for the next chunk of it
        _read("read_64k", [65536], [65536], 8, 8),
        # sequences taken out of a paged server cache
        _read("read_paged_ragged", [30011, 1, 12289, 4096], [30011, 1, 12289, 4096], 8, 4, page=16),
        # a short chat turn of a small model: latency counts
        _decode("decode_short", [700], 8, 2, 8),
        # a decode batch of mixed lengths, capped scores with a distance bias
        _decode("decode_ragged_cap", [32768, 5001, 77777, 20480, 1, 12289], 32, 8, 8, cap=50, alibi=True),
        # long contexts at four bits
        _decode("decode_128k_b4", [131072] * 4, 32, 8, 4),
        # a server's batch over pages, eight heads to a KV head
        _decode("decode_paged_16", [4000 + 640 * i for i in range(16)], 64, 8, 8, page=64),
        # which blocks of a few short sequences a token looks at
        _chosen("select_short", "select", [3000, 801], 8, 2, 8, 16, 32),
        # the same of long ones
        _chosen("select_128k_b4", "select", [131072] * 4, 32, 8, 4, 64, 128),
        # one step over a sixteenth of long contexts
        _chosen("blocks_128k_b4", "blocks", [131072] * 4, 32, 8, 4, 64, 128),
        # one step at a million tokens, in pages
        _chosen("blocks_1m_paged", "blocks", [1048576], 32, 8, 8, 128, 64, page=128),
    ]


def draw(rng):
    def size(lo, hi):
        lo, hi = max(1, int(lo)), max(1, int(lo), int(hi))
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n if rng.random() < 0.7 or n < 128 else max(lo, n // 64 * 64)

    op = rng.choice(["write", "read", "decode", "decode", "decode", "select", "blocks", "blocks"])
    hq, hkv = rng.choice([(8, 2), (32, 8), (32, 8), (64, 8), (16, 8), (8, 8)])
    bits, page = rng.choice([8, 4]), rng.choice([0, 0, 16, 64, 50])
    nb = int(round(math.exp(rng.uniform(0, math.log(32)))))
    if op in ("write", "read"):
        step = rng.random() < 0.4
        lens = [size(1, (8192 if step else 60000 / nb)) for _ in range(nb)]
        new = [1 if step else size(1, n) if rng.random() < 0.4 else n for n in lens]
        if op == "write":
            return {k: v for k, v in _write("", lens, new, hkv, bits, page, rng.choice([0, 16, 32, 64, 128])).items() if k != "name"}
        return {k: v for k, v in _read("", lens, new, hkv, bits, page).items() if k != "name"}
    lens = [size(1, 250000 / nb) for _ in range(nb)]
    if op == "decode":
        c = _decode("", lens, hq, hkv, bits, page, rng.choice([0, 0, 30, 50]), rng.random() < 0.4)
    else:
        first, last = rng.choice([0, 1, 4]), rng.choice([1, 2, 8])
        c = _chosen("", op, lens, hq, hkv, bits, rng.choice([16, 32, 64, 128]), max(first + last, size(4, 300)), page, first, last)
    c.pop("name")
    return c


# ------------------------------------------------------------------------------------------ the format
def _powers(x, bits):
    """Exponents of the groups of x [..][128], 32 bits: the least whose largest value is not below the group's."""
    top = x.unflatten(-1, (4, 32)).abs().amax(-1)
    m, e = torch.frexp(top)  # top = m 2^e, m in [1/2, 1)
    full, ehi = (0.875, 9) if bits == 8 else (0.75, 3)  # 448 = 0.875 2^9, 6 = 0.75 2^3
    s = torch.where(top > 0, e - ehi + (m > full), -200)
    return s.clamp(-117, 119) if bits == 8 else s.clamp(-125, 125)


def _encode(x, bits):
    """Codes uint8 [..][16 bits] and scales uint8 [..][4] of x bf16 [..][128]."""
    x = x.float()
    s = _powers(x, bits)
    y = torch.ldexp(x.unflatten(-1, (4, 32)), -s[..., None]).flatten(-2)
    scales = (s + 127).to(torch.uint8)
    if bits == 8:
        return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), scales
    a = y.abs().clamp(max=6)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step  # (ties to even)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., ::2] | (code[..., 1::2] << 4), scales


def _decode_values(codes, scales, bits):
    """Values in 32 bits of codes and scales."""
    if bits == 8:
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(torch.int64)
        v = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)[c]
    return torch.ldexp(v.unflatten(-1, (4, 32)), scales.to(torch.int32)[..., None] - 127).flatten(-2)


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + stream)
    return g


def _tokens(gen, hkv, n):
    """bf16 [hkv][n][128]: runs of tokens about one subject, some dimensions larger than others."""
    width = torch.exp(0.5 * torch.randn(hkv, 1, D, generator=gen, device=DEV))
    subject = torch.randn(hkv, n // 96 + 1, D, generator=gen, device=DEV).to(torch.bfloat16)
    x = torch.empty(hkv, n, D, dtype=torch.bfloat16, device=DEV)
    for i in range(0, n, 1 << 18):
        j = min(n, i + (1 << 18))
        at = torch.arange(i, j, device=DEV) // 96
        x[:, i:j] = ((torch.randn(hkv, j - i, D, generator=gen, device=DEV) + subject[:, at].float()) * (0.7 * width)).to(torch.bfloat16)
    return x


def _starts(case):
    """First row of every sequence's span, and all rows."""
    ends = np.cumsum([0] + [n + SPARE for n in _ints(case["lens"])])
    return [int(x) for x in ends[:-1]], int(ends[-1])


def _places(case, seed):
    """The page table (None: spans) and, for each sequence, the place of every row: its row of [hkv][total], or page times
    page size plus the row of the page in [pages][hkv][page], the pages in shuffled order."""
    lens, page = _ints(case["lens"]), case["page"]
    if not page:
        return None, [torch.arange(a, a + n, device=DEV) for a, n in zip(_starts(case)[0], lens)]
    counts = [max(1, -(-(n + SPARE) // page)) for n in lens]
    place = torch.as_tensor(np.random.default_rng([int(seed), 7]).permutation(sum(counts)).astype(np.int32), device=DEV)
    table = torch.zeros(len(lens), max(counts), dtype=torch.int32, device=DEV)
    for b, ids in enumerate(place.split(counts)):
        table[b, :len(ids)] = ids
    return table, [table[b].long().repeat_interleave(page)[:n] * page + torch.arange(n, device=DEV) % page for b, n in enumerate(lens)]


def _get(x, rows, page):
    """Rows (places) of every head: [hkv][len(rows)][..]."""
    return x[:, rows] if not page else x[rows // page, :, rows % page].transpose(0, 1)


def _put(x, rows, page, values):
    if page:
        x[rows // page, :, rows % page] = values.transpose(0, 1)
    else:
        x[:, rows] = values


def _inputs(case, seed):
    """Everything a call reads: the cache's arrays with its rows, the tokens to write, the queries."""
    lens, hkv, hq, bits, page, block = _ints(case["lens"]), case["hkv"], case["hq"], case["bits"], case["page"], case["block"]
    gen, total = _gen(seed, 1), _starts(case)[1]
    table, places = _places(case, seed)
    shape = (hkv, total) if not page else (sum(max(1, -(-(n + SPARE) // page)) for n in lens), hkv, page)
    s = dict(case=case, lens=lens, places=places, table=table)
    for name in ("K", "V"):
        s[name] = torch.zeros(*shape, 16 * bits, dtype=torch.uint8, device=DEV)
        s[name + "_scale"] = torch.full((*shape, 4), 127, dtype=torch.uint8, device=DEV)
    s["bounds"] = torch.zeros(hkv, total // block + len(lens), 2, D, dtype=torch.bfloat16, device=DEV) if block else None
    new = _ints(case.get("new", ""))
    if case["op"] == "write":
        s["k"], s["v"] = (_tokens(gen, hkv, sum(new)).transpose(0, 1).contiguous() for _ in range(2))
    for b, n in enumerate(lens):
        had = n - new[b] if case["op"] == "write" else n
        for i in range(0, had, 1 << 18):
            rows = places[b][i:min(had, i + (1 << 18))]
            for name in ("K", "V"):
                codes, scales = _encode(_tokens(gen, hkv, len(rows)), bits)
                _put(s[name], rows, page, codes)
                _put(s[name + "_scale"], rows, page, scales)
    new = new or [0] * len(lens)
    if block:
        _bound(s, _touched(s, [0] * len(lens), [n - m for n, m in zip(lens, new)] if case["op"] == "write" else lens))
        s["touched"] = _touched(s, [n - m for n, m in zip(lens, new)], lens)
    s["last"] = torch.cat([p[len(p) - m:] for p, m in zip(places, new)])
    s["slopes"] = (torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=DEV)
                   if case.get("alibi") else None)
    s["q"] = (1.5 * torch.randn(len(lens), hq, D, generator=gen, device=DEV)).to(torch.bfloat16)
    return s


def _touched(s, begins, ends):
    """The blocks from that of row begins[b] to that of row ends[b] - 1 of every sequence: their places in the bounds, the
    places of their rows [blocks][L], and which of these rows there are."""
    L, slots, rows, held = s["case"]["block"], [], [], []
    for b, (i, j) in enumerate(zip(begins, ends)):
        blocks = torch.arange(i // L, -(-j // L) if j > i else i // L, device=DEV)
        r = blocks[:, None] * L + torch.arange(L, device=DEV)
        slots.append(_starts(s["case"])[0][b] // L + b + blocks)
        rows.append(s["places"][b][r.clamp(max=max(0, j - 1))])
        held.append(r < j)
    return torch.cat(slots), torch.cat(rows), torch.cat(held)


def _bound(s, touched):
    """Sets the bounds of such blocks."""
    case, page = s["case"], s["case"]["page"]
    for slots, rows, held in zip(*(x.split(1 << 12) for x in touched)):
        k = _decode_values(*(_get(s[x], rows.flatten(), page) for x in ("K", "K_scale")), case["bits"]).unflatten(1, rows.shape)
        lo, hi = (k.masked_fill(~held[None, :, :, None], sign * math.inf) for sign in (1, -1))
        s["bounds"][:, slots] = torch.stack([lo.amin(2), hi.amax(2)], 2).to(torch.bfloat16)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2502_12216_amd as T
        batch = T.RaggedBatch(s["lens"], case["hq"], case["hkv"], capacities=[n + SPARE for n in s["lens"]])
        s["batch"] = batch
        s["cache"] = T.QuantizedCache(s["K"], s["K_scale"], s["V"], s["V_scale"], bounds=s["bounds"], block=case["block"],
                                      page_table=s["table"])
        if case["op"] in ("write", "read"):
            s["rows"] = T.CacheQuantizer(batch, _ints(case["new"]))
        if case["op"] in ("select", "blocks"):
            s["select"] = T.BlockSelector(batch, case["block"], case["budget"], first=case["first"], last=case["last"])
        if case["op"] in ("decode", "blocks"):
            s["decoder"] = T.QuantizedDecoder(batch)
            s["mod"] = T.ScoreMod(cap=case["cap"], slopes=s["slopes"])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"write": _plain_write, "read": _plain_read, "decode": _plain_decode, "select": _plain_select,
            "blocks": _plain_blocks}[state["case"]["op"]](state)


def _run_own(s):
    op = s["case"]["op"]
    if op == "write":
        s["rows"].write(s["k"], s["v"], s["cache"])
        K, V = s["rows"].read(s["cache"])
        return {"K": K, "V": V, "bounds": s["bounds"]} if s["case"]["block"] else {"K": K, "V": V}
    if op == "read":
        K, V = s["rows"].read(s["cache"])
        return {"K": K, "V": V}
    if op == "decode":
        out, lse = s["decoder"](s["q"], s["cache"], s["mod"])
        return {"out": out, "lse": lse}
    blocks, counts = s["select"](s["q"], s["cache"])
    if op == "select":
        return {"blocks": blocks, "counts": counts}
    out, lse = s["decoder"](s["q"], s["cache"], s["mod"], blocks=blocks, counts=counts)
    return {"blocks": blocks, "counts": counts, "out": out, "lse": lse}


# ------------------------------------------------------------------------------------------ the plain forms
def _values(s, name, rows):
    """Values in 32 bits [hkv][len(rows)][128] of places of the cache."""
    page = s["case"]["page"]
    return _decode_values(_get(s[name], rows, page), _get(s[name + "_scale"], rows, page), s["case"]["bits"])


def _plain_read(s):
    rows = s["last"]
    return {"K": _values(s, "K", rows).to(torch.bfloat16), "V": _values(s, "V", rows).to(torch.bfloat16)}


def _plain_write(s):
    rows, case = s["last"], s["case"]
    for name, x in (("K", s["k"]), ("V", s["v"])):
        codes, scales = _encode(x.transpose(0, 1), case["bits"])
        _put(s[name], rows, case["page"], codes)
        _put(s[name + "_scale"], rows, case["page"], scales)
    got = _plain_read(s)
    if not case["block"]:
        return got
    _bound(s, s["touched"])
    return dict(got, bounds=s["bounds"])


def _attend(s, q, k, v, distance, seen):
    """out [..][G][128], lse [..][G] of q [..][G][128] over k, v [..][n][128], all 32 bits; distance [..][n]; seen [..][n] or None."""
    case = s["case"]
    z = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(D)
    if case["cap"]:
        z = case["cap"] * torch.tanh(z / case["cap"])
    if s["slopes"] is not None:
        z = z - s["slopes"].view(case["hkv"], -1, 1) * distance.unsqueeze(-2)
    if seen is not None:
        z = z.masked_fill(~seen.unsqueeze(-2), -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v) / total, (torch.log(total) + top)[..., 0]


def _plain_decode(s):
    case, got = s["case"], []
    q = s["q"].float().unflatten(1, (case["hkv"], -1))
    for b, n in enumerate(s["lens"]):
        k, v = (_values(s, name, s["places"][b]) for name in ("K", "V"))
        got.append(_attend(s, q[b], k, v, torch.arange(n - 1, -1, -1, device=DEV), None))
    return {"out": torch.stack([x[0].flatten(0, 1) for x in got]), "lse": torch.stack([x[1].flatten() for x in got])}


def _plain_select(s):
    case, L = s["case"], s["case"]["block"]
    B, hkv, budget = len(s["lens"]), case["hkv"], case["budget"]
    q = s["q"].double().unflatten(1, (hkv, -1))
    blocks = torch.full((B, hkv, budget), -1, dtype=torch.int32, device=DEV)
    counts = torch.zeros(B, hkv, dtype=torch.int32, device=DEV)
    for b, (n, a) in enumerate(zip(s["lens"], _starts(case)[0])):
        nb = -(-n // L)
        lo, hi = s["bounds"][:, a // L + b:a // L + b + nb].double().unbind(2)
        u = (torch.matmul(q[b].clamp(min=0), hi.transpose(1, 2).contiguous()) +
             torch.matmul(q[b].clamp(max=0), lo.transpose(1, 2).contiguous()))
        score = (u - u.amax(2, keepdim=True)).amax(1)
        score[:, :case["first"]] = math.inf
        score[:, max(0, nb - case["last"]):] = math.inf
        k = min(budget, nb)
        best = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :k]
        blocks[b, :, :k] = torch.sort(best, dim=1).values.to(torch.int32)
        counts[b] = k
    return {"blocks": blocks, "counts": counts}


def _plain_blocks(s):
    case, L, page = s["case"], s["case"]["block"], s["case"]["page"]
    hkv, got = case["hkv"], _plain_select(s)
    q, outs = s["q"].float().unflatten(1, (hkv, -1)), []
    heads = torch.arange(hkv, device=DEV)[:, None]
    for b, n in enumerate(s["lens"]):
        row = (got["blocks"][b].long()[:, :, None] * L + torch.arange(L, device=DEV)).flatten(1)
        seen = (row >= 0) & (row < n)
        place = s["places"][b][row.clamp(0, n - 1)]
        k, v = (_decode_values(*((x[heads, place] if not page else x[place // page, heads, place % page])
                                 for x in (s[name], s[name + "_scale"])), case["bits"]) for name in ("K", "V"))
        outs.append(_attend(s, q[b], k, v, n - 1 - row, seen))
    return dict(got, out=torch.stack([x[0].flatten(0, 1) for x in outs]), lse=torch.stack([x[1].flatten() for x in outs]))


# ------------------------------------------------------------------------------------------ what a call cannot do without
def work(case):
    lens, hq, hkv, L = _ints(case["lens"]), case["hq"], case["hkv"], case["block"]
    row = 16 * case["bits"] + 4
    if case["op"] in ("write", "read"):
        new = sum(_ints(case["new"]))
        size = new * hkv * 2 * (row + 2 * D)
        if case["op"] == "write":  # in and out, the blocks' rows before the new ones, and the values stored back in bf16
            size += size
            if L:
                touched = sum(-(-n // L) - (n - m) // L for n, m in zip(lens, _ints(case["new"])))
                before = sum((n - m) % L for n, m in zip(lens, _ints(case["new"])))
                size += hkv * (touched * 4 * D + before * row)
        return {"bytes": size, "flops": 4.0 * new * hkv * D}
    ends = len(lens) * hq * (2 * D + 4 * D + 4)
    if case["op"] == "decode":
        return {"bytes": sum(lens) * hkv * 2 * row + ends, "flops": 4.0 * D * hq * sum(lens)}
    nb = [-(-n // L) for n in lens]
    size, flops = sum(nb) * hkv * 4 * D + len(lens) * (hq * 2 * D + hkv * 4 * (case["budget"] + 1)), 4.0 * D * hq * sum(nb)
    if case["op"] == "blocks":
        held = sum(min(n, case["budget"] * L) for n in lens)
        size, flops = size + held * hkv * 2 * row + ends, flops + 4.0 * D * hq * held
    return {"bytes": size, "flops": flops}


# ------------------------------------------------------------------------------------------ the same in 64 bits
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_stored(x, bits):
    """What a cache of `bits` bits holds of x [..][128], in 64 bits."""
    x = x.double().reshape(*x.shape[:-1], 4, 32)
    largest = 448.0 if bits == 8 else 6.0
    amax = x.abs().max(-1, keepdim=True).values
    s = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -150) / largest))
    s = torch.where(amax <= largest * torch.exp2(s - 1), s - 1, s)  # (the logarithm's own rounding)
    s = torch.where(amax > largest * torch.exp2(s), s + 1, s)
    s = s.clamp(-117, 119) if bits == 8 else s.clamp(-125, 125)
    y = (x * torch.exp2(-s)).clamp(-largest, largest)
    binade = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -30))).clamp(min=-6 if bits == 8 else 0)
    ulp = torch.exp2(binade - (3 if bits == 8 else 1))
    return (torch.round(y / ulp) * ulp * torch.exp2(s)).reshape(*x.shape[:-2], D)


def _exact_held(s, name, b, g, rows):
    """Rows of head g of sequence b in 64 bits, from the codes."""
    case, place = s["case"], s["places"][b][rows]
    page = case["page"]
    at = (place // page, g, place % page) if page else (g, place)
    codes, power = s[name][at].to(torch.int64), s[name + "_scale"][at].double() - 127
    if case["bits"] == 8:
        e, m = (codes >> 3) & 15, (codes & 7).double()
        v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e.double() - 7)) * (1 - 2.0 * (codes >> 7))
    else:
        c = torch.empty(len(codes), D, dtype=torch.int64, device=DEV)
        c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
        v = torch.tensor(E2M1, dtype=torch.float64, device=DEV)[c & 7] * (1 - 2.0 * (c >> 3))
    return v * torch.exp2(power).repeat_interleave(32, dim=1)


def _exact_head(case, q, k, v, slope, distance):
    x = (k @ q) * D ** -0.5
    if case["cap"]:
        x = torch.tanh(x / case["cap"]) * case["cap"]
    if slope is not None:
        x = x - slope.double() * distance
    lse = torch.logsumexp(x, 0)
    return torch.exp(x - lse) @ v, lse


def exact(case, seed):
    s = _inputs(case, seed)
    lens, hq, hkv, L = s["lens"], case["hq"], case["hkv"], case["block"]
    B, G = len(lens), hq // hkv
    if case["op"] == "read":
        got = [torch.cat([torch.stack([_exact_held(s, x, b, g, torch.arange(n - m, n, device=DEV)) for g in range(hkv)])
                          for b, (n, m) in enumerate(zip(lens, _ints(case["new"])))], 1) for x in ("K", "V")]
        return {"K": got[0], "V": got[1]}
    if case["op"] == "write":
        K, V = (_exact_stored(s[x], case["bits"]).transpose(0, 1) for x in ("k", "v"))
        if not L:
            return {"K": K, "V": V}
        bounds, at = s["bounds"].double(), 0
        for b, (n, m) in enumerate(zip(lens, _ints(case["new"]))):
            first, lead = _starts(case)[0][b] // L + b, (n - m) % L
            for g in range(hkv):
                rows = torch.cat([_exact_held(s, "K", b, g, torch.arange(n - m - lead, n - m, device=DEV)), K[g, at:at + m]])
                full = len(rows) // L * L
                parts = [rows[:full].reshape(-1, L, D)] + ([rows[full:][None]] if len(rows) > full else [])
                to = first + (n - m) // L
                for p in parts:
                    bounds[g, to:to + len(p), 0], bounds[g, to:to + len(p), 1] = p.min(1).values, p.max(1).values
                    to += len(p)
            at += m
        return {"K": K, "V": V, "bounds": bounds}
    out = torch.zeros(B, hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, hq, dtype=torch.float64, device=DEV)
    blocks = torch.full((B, hkv, case.get("budget", 0)), -1, dtype=torch.int32, device=DEV)
    counts = torch.zeros(B, hkv, dtype=torch.int32, device=DEV)
    for b, n in enumerate(lens):
        for g in range(hkv):
            rows = torch.arange(n, device=DEV)
            if L:
                rows = _exact_choice(s, b, g)
                blocks[b, g, :len(rows)], counts[b, g] = rows, len(rows)
                if case["op"] == "select":
                    continue
                rows = torch.cat([torch.arange(j * L, min(n, j * L + L), device=DEV) for j in rows.tolist()])
            k, v = _exact_held(s, "K", b, g, rows), _exact_held(s, "V", b, g, rows)
            for h in range(g * G, g * G + G):
                out[b, h], lse[b, h] = _exact_head(case, s["q"][b, h].double(), k, v, None if s["slopes"] is None else s["slopes"][h],
                                                   (n - 1 - rows).double())
    if case["op"] == "select":
        return {"blocks": blocks, "counts": counts}
    return {"blocks": blocks, "counts": counts, "out": out, "lse": lse} if L else {"out": out, "lse": lse}


def _exact_choice(s, b, g):
    """The chosen blocks of head g of sequence b, ascending, ranked on the host."""
    case, n, L = s["case"], s["lens"][b], s["case"]["block"]
    nb, G = -(-n // L), case["hq"] // case["hkv"]
    at = _starts(case)[0][b] // L + b
    lo, hi = (s["bounds"][g, at:at + nb, i].double().cpu().numpy() for i in (0, 1))
    score = np.full(nb, -np.inf)
    for h in range(g * G, g * G + G):
        q = s["q"][b, h].double().cpu().numpy()
        u = np.maximum(q * lo, q * hi).sum(1)
        score = np.maximum(score, u - u.max())
    i = np.arange(nb)
    always = (i < case["first"]) | (i >= nb - case["last"])
    order = np.lexsort((i, -score, ~always))
    return torch.as_tensor(np.sort(order[:case["budget"]]).astype(np.int32), device=DEV)
