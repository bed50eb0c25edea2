"""The attention and cache operators beside the dense decode: their calls, inputs, plain forms and 64-bit results.

A case is a dict of plain values.  `op` names the entry point:

  prompt    PromptAttention(...)      attention of each sequence's last `new` tokens over its cache, causal, with
                                      capped scores, a distance bias, documents or a prefix that all tokens see
  decode    ScoredDecoder(...)        one token per sequence with the same scores, over a cache that may hold any
                                      positions, and the attention weights added to a running sum per cached row
  shared    SharedPrefixDecoder(...)  one token per sequence; several sequences share the keys of a long prefix
  weights   PromptAttention.add_weights  the attention weights that the last queries give to every cached row
  evict     CacheEvictor(...)         keeps the recent rows and those of the largest weights, in another cache
  insert    TokenInserter(...)        a new token per sequence into a full cache, in place of the least one

`page` > 0 reads the cache through pages of so many tokens (.paged).  Lists of numbers are comma-separated texts.
"""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128
DEV = "cuda"
own = False


# ------------------------------------------------------------------------------------------ the cases
def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _text(values):
    return ",".join(str(int(x)) for x in values)


def _scores_of(cap=0.0, alibi=False, docs=0, prefix=False):
    return dict(cap=float(cap), alibi=alibi, docs=docs, prefix=prefix)


def _prompt(name, lens, new, hq, hkv, page=0, **kw):
    return dict(name=name, op="prompt", lens=_text(lens), new=_text(new), hq=hq, hkv=hkv, page=page, **_scores_of(**kw))


def _decode(name, lens, hq, hkv, page=0, evicted=False, add=False, **kw):
    return dict(name=name, op="decode", lens=_text(lens), hq=hq, hkv=hkv, page=page, evicted=evicted, add=add,
                **_scores_of(**kw))


def _shared(name, prefixes, of, lens, hq, hkv, page=0, **kw):
    return dict(name=name, op="shared", prefixes=_text(prefixes), of=_text(of), lens=_text(lens), hq=hq, hkv=hkv,
                page=page, **_scores_of(**kw))


def _weights(name, lens, new, window, hq, hkv, **kw):
    return dict(name=name, op="weights", lens=_text(lens), new=_text(new), window=window, hq=hq, hkv=hkv, page=0,
                **_scores_of(**kw))


def _evict(name, lens, keep, recent, hkv):
    return dict(name=name, op="evict", lens=_text(lens), keep=_text(keep), recent=recent, hq=hkv, hkv=hkv)


def _insert(name, lens, recent, hkv):
    return dict(name=name, op="insert", lens=_text(lens), recent=recent, hq=hkv, hkv=hkv)


def listed():
    tails = [(137 * i * i + 61 * i) % 1900 + 1 for i in range(32)]
    return [
        # a short chat turn of a small model: latency counts
        _prompt("prompt_short_cap", [211], [211], 8, 2, cap=30),
        # one chunk of a long prompt, against the paged cache of the chunks before it
        _prompt("prompt_chunk_paged", [65536], [512], 32, 8, page=64, alibi=True),
        # a prefill batch whose sequences are packed with documents of many lengths
        _prompt("prompt_documents", [16000, 8192, 5001], [16000, 8192, 5001], 32, 8, cap=50, docs=1100),
        # a long prompt whose first tokens (the instructions) all tokens see
        _prompt("prompt_16k_prefix", [16384], [16384], 32, 8, alibi=True, prefix=True),
        # a decode batch of mixed lengths, capped scores with a distance bias
        _decode("decode_ragged_cap", [32768, 5001, 77777, 20480, 1, 12289], 32, 8, cap=50, alibi=True),
        # one step over caches that eviction holds at 2048 rows, summing the weights the next eviction goes by
        _decode("decode_evicted_sum", [2048] * 16, 32, 8, evicted=True, add=True, alibi=True),
        # four samples of one prompt, a few tokens in
        _shared("shared_4_samples", [4096], [0] * 4, [3, 9, 17, 40], 8, 2),
        # a server's system prompt and documents before 32 conversations
        _shared("shared_32_chats", [32768], [0] * 32, tails, 32, 8),
        # which rows the last queries of a long prompt look at (before a prompt's cache is compressed)
        _weights("weights_last_64", [65536, 20001], [64, 64], 64, 32, 8),
        # the same over every query of a prompt
        _weights("weights_all_8k", [8192], [8192], 0, 32, 8, cap=50),
        # a prompt's cache compressed to a quarter
        _evict("evict_64k", [65536, 30011], [16384, 7500], 512, 8),
        # a decode step's new token into full caches
        _insert("insert_full_16", [2048] * 16, 256, 8),
    ]


def draw(rng):
    def size(lo, hi):
        lo, hi = max(1, int(lo)), max(1, int(lo), int(hi))
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n if rng.random() < 0.7 or n < 128 else max(lo, n // 64 * 64)

    op = rng.choice(["prompt", "prompt", "decode", "decode", "shared", "shared", "weights", "evict", "insert"])
    hq, hkv = rng.choice([(8, 2), (32, 8), (32, 8), (64, 8), (16, 8), (8, 8)])
    kw = dict(cap=rng.choice([0, 0, 30, 50]), alibi=rng.random() < 0.4)
    if op == "prompt":
        nb = rng.choice([1, 1, 2, 3])
        new = [size(1, 8192 * math.sqrt(8 / hq / nb) if hq > 8 else 8192 / nb) for _ in range(nb)]
        lens = [m + (size(1, 40000) if rng.random() < 0.4 else 0) for m in new]
        kw.update(docs=rng.choice([0, 0, 300, 2000]), prefix=rng.random() < 0.25)
        c = _prompt("", lens, new, hq, hkv, page=rng.choice([0, 0, 16, 64]), **kw)
    elif op == "decode":
        nb = int(round(math.exp(rng.uniform(0, math.log(24)))))
        evicted = rng.random() < 0.4
        lens = [size(1, 8192 if evicted else 200000 / nb) for _ in range(nb)]
        kw.update(docs=rng.choice([0, 0, 900]) if not evicted else 0)
        c = _decode("", lens, hq, hkv, page=0 if evicted else rng.choice([0, 0, 16, 64]), evicted=evicted,
                    add=rng.random() < 0.5, **kw)
    elif op == "shared":
        np_, nb = rng.choice([1, 1, 2, 3]), int(round(math.exp(rng.uniform(math.log(2), math.log(48)))))
        c = _shared("", [size(16, 60000 / np_) for _ in range(np_)], [rng.randrange(-1 if nb > 4 else 0, np_) for _ in range(nb)],
                    [size(1, 3000) for _ in range(nb)], hq, hkv, page=rng.choice([0, 0, 16, 64]), **kw)
    elif op == "weights":
        nb = rng.choice([1, 1, 2])
        if rng.random() < 0.5:
            new = [size(1, 200) for _ in range(nb)]
            lens = [m + size(100, 60000) for m in new]
        else:
            new = lens = [size(64, 5000 / nb) for _ in range(nb)]
        c = _weights("", lens, new, rng.choice([0, 0, 16, 100]), hq, hkv, **kw)
    elif op == "evict":
        lens = [size(64, 90000) for _ in range(rng.choice([1, 1, 2, 4]))]
        c = _evict("", lens, [size(8, n) for n in lens], rng.choice([0, 1, 64, 500]), hkv)
    else:
        c = _insert("", [size(8, 16384)] * int(round(math.exp(rng.uniform(0, math.log(32))))), rng.choice([0, 1, 64, 300]), hkv)
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(np.random.SeedSequence([int(seed), int(tag)]).generate_state(1, dtype=np.uint64)[0] >> 1))
    return g


def _randn(gen, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * scale).to(torch.bfloat16)


def _slopes(hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=DEV)


def _documents(n, mean):
    """Document of each of n tokens: runs of lengths around `mean`, the same for every seed."""
    cuts = np.random.default_rng([n, mean]).exponential(mean, size=4 * n // mean + 8).astype(np.int64).cumsum()
    return np.searchsorted(cuts, np.arange(n), side="right").astype(np.int32)


def _prefix_len(new):
    return max(1, new // 16)


def _inputs(case, seed):
    """Everything a call reads; K and V in token order."""
    lens, hkv, hq = _ints(case["lens"]), case["hkv"], case["hq"]
    gen, total, B = _gen(seed, 1), sum(lens), len(lens)
    s = dict(case=case, lens=lens)
    s["K"], s["V"] = _randn(gen, hkv, total, D), _randn(gen, hkv, total, D)
    if case["op"] in ("evict", "insert"):
        # sums of attention weights: a few large ones, many small, some rows never looked at
        w = torch.rand(hkv, total, generator=gen, device=DEV).clamp_min(1e-6) ** -0.7 - 1.0
        s["weights"] = torch.where(torch.rand(hkv, total, generator=gen, device=DEV) < 0.05, 0.0, w)
        s["positions"] = _spread_positions(gen, lens, hkv)
        s["keep"] = torch.tensor(_ints(case.get("keep", "")), dtype=torch.int32, device=DEV)
        s["k"], s["v"] = _randn(gen, B, hkv, D), _randn(gen, B, hkv, D)
        newest = [int(x[-1]) for x in s["positions"][0].split(lens)]
        s["newest"] = torch.tensor([x + (case["op"] == "insert") for x in newest], dtype=torch.int32, device=DEV)
        return s
    s["slopes"] = _slopes(hq) if case["alibi"] else None
    s["documents"] = s["prefix_len"] = s["q_documents"] = None
    if case["docs"]:
        docs = [_documents(n, case["docs"]) for n in lens]
        s["documents"] = torch.as_tensor(np.concatenate(docs), device=DEV)
        s["q_documents"] = torch.tensor([int(d[-1]) for d in docs], dtype=torch.int32, device=DEV)
    if case["op"] in ("prompt", "weights"):
        new = _ints(case["new"])
        s["new"] = new
        s["q"] = _randn(gen, sum(new), hq, D, scale=2.0)
        if case["prefix"]:
            s["prefix_len"] = torch.tensor([n - m + _prefix_len(m) for n, m in zip(lens, new)], dtype=torch.int32, device=DEV)
    else:
        s["q"] = _randn(gen, B, hq, D, scale=2.0)
    if case["op"] == "weights":
        s["lse"] = torch.cat([x[1] for x in _every_query(s)], 1)
        s["sums"] = torch.rand(hkv, total, generator=gen, device=DEV)
    if case["op"] == "decode":
        s["positions"] = _spread_positions(gen, lens, hkv) if case["evicted"] else None
        s["q_pos"] = None
        if case["evicted"]:
            s["q_pos"] = torch.stack([x[-1] for x in s["positions"][0].split(lens)]).contiguous()
        s["sums"] = torch.rand(hkv, total, generator=gen, device=DEV) if case["add"] else None
    if case["op"] == "shared":
        s["prefixes"], s["of"] = _ints(case["prefixes"]), _ints(case["of"])
        s["Kp"], s["Vp"] = _randn(gen, hkv, sum(s["prefixes"]), D), _randn(gen, hkv, sum(s["prefixes"]), D)
    return s


def _spread_positions(gen, lens, hkv):
    """Positions of cached rows after evictions: ascending, with gaps, the newest the same for every head."""
    out = []
    for n in lens:
        p = torch.cumsum(torch.randint(1, 6, (hkv, n), generator=gen, device=DEV, dtype=torch.int32), 1, dtype=torch.int32)
        out.append(p + (p[:, -1].max() - p[:, -1:]))
    return torch.cat(out, 1).contiguous()


def _paged(x, lens, page, seed):
    """Pages [pages][hkv][page][128] of x [hkv][total][128], in shuffled places, and the page table."""
    counts = [max(1, -(-n // page)) for n in lens]
    place = torch.as_tensor(np.random.default_rng([int(seed), 7]).permutation(sum(counts)).astype(np.int32), device=DEV)
    table = torch.zeros(len(lens), max(counts), dtype=torch.int32, device=DEV)
    pages = torch.zeros(sum(counts), x.shape[0], page, D, dtype=x.dtype, device=DEV)
    for b, (ids, rows) in enumerate(zip(place.split(counts), x.split(lens, 1))):
        table[b, :len(ids)] = ids
        rows = torch.nn.functional.pad(rows, (0, 0, 0, len(ids) * page - rows.shape[1]))
        pages[ids.long()] = rows.unflatten(1, (len(ids), page)).transpose(0, 1)
    return pages, table


def prepare(case, seed):
    s = _inputs(case, seed)
    op, lens, page = case["op"], s["lens"], case.get("page", 0)
    if page:
        s["Kpg"], s["table"] = _paged(s["K"], lens, page, seed)
        s["Vpg"], _ = _paged(s["V"], lens, page, seed)
        if op == "shared":
            s["Kppg"], s["ptable"] = _paged(s["Kp"], s["prefixes"], page, seed)
            s["Vppg"], _ = _paged(s["Vp"], s["prefixes"], page, seed)
    if op in ("evict", "insert"):
        kept = [min(n, k) for n, k in zip(lens, _ints(case.get("keep", "")))]
        room = sum(kept)
        s["kept"] = kept
        s["K_out"], s["V_out"] = (torch.zeros(case["hkv"], room, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        s["weights_out"] = torch.zeros(case["hkv"], room, device=DEV)
        s["positions_out"] = torch.zeros(case["hkv"], room, dtype=torch.int32, device=DEV)
        s["seq_len"] = torch.tensor(lens, device=DEV)
    if own:
        import paper_2502_12216_amd as T
        hq, hkv = case["hq"], case["hkv"]
        if op == "insert":
            s["batch"] = T.RaggedBatch(lens, hq, hkv, capacities=lens)
            s["call"] = T.TokenInserter(s["batch"], case["recent"])
            return s
        batch = T.RaggedBatch(lens, hq, hkv)
        if op == "evict":
            s["dest"] = T.RaggedBatch([0] * len(lens), hq, hkv, capacities=s["kept"])
            s["call"] = T.CacheEvictor(batch, s["dest"], case["recent"])
            return s
        s["mod"] = T.ScoreMod(cap=case["cap"], slopes=s["slopes"], documents=s["documents"], prefix_len=s["prefix_len"])
        s["call"] = (T.PromptAttention(batch, s["new"]) if op in ("prompt", "weights") else T.ScoredDecoder(batch)
                     if op == "decode" else T.SharedPrefixDecoder(batch, s["prefixes"], s["of"]))
        if page:
            s["cache"] = T.PagedCache(s["Kpg"], s["Vpg"], s["table"])
            if op == "shared":
                s["pcache"] = T.PagedCache(s["Kppg"], s["Vppg"], s["ptable"])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"prompt": _plain_prompt, "decode": _plain_decode, "shared": _plain_shared, "weights": _plain_weights,
            "evict": _plain_evict, "insert": _plain_insert}[state["case"]["op"]](state)


def _run_own(s):
    op, page, call = s["case"]["op"], s["case"].get("page", 0), s["call"]
    if op == "prompt":
        out, lse = call.paged(s["q"], s["cache"], s["mod"]) if page else call(s["q"], s["K"], s["V"], s["mod"])
        return {"out": out, "lse": lse}
    if op == "decode":
        more = dict(positions=s["positions"], q_pos=s["q_pos"], q_documents=s["q_documents"], weights=s["sums"])
        out, lse = call.paged(s["q"], s["cache"], s["mod"], **more) if page else call(s["q"], s["K"], s["V"], s["mod"], **more)
        return {"out": out, "lse": lse, "sums": s["sums"]} if s["case"]["add"] else {"out": out, "lse": lse}
    if op == "shared":
        out, lse = (call.paged(s["q"], s["pcache"], s["cache"], s["mod"]) if page else
                    call(s["q"], s["Kp"], s["Vp"], s["K"], s["V"], s["mod"]))
        return {"out": out, "lse": lse}
    if op == "weights":
        return {"sums": call.add_weights(s["q"], s["K"], s["lse"], s["sums"], s["mod"], window=s["case"]["window"])}
    if op == "evict":
        call(s["K"], s["V"], s["weights"], s["keep"], s["K_out"], s["V_out"], s["weights_out"], s["positions_out"],
             positions=s["positions"], newest=s["newest"])
        return {"K": s["K_out"], "V": s["V_out"], "weights": s["weights_out"], "positions": s["positions_out"],
                "lens": s["dest"].seq_len}
    row = call(s["k"], s["v"], s["K"], s["V"], s["weights"], s["positions"], s["newest"])
    return {"row": row, "K": s["K"], "V": s["V"], "weights": s["weights"], "positions": s["positions"],
            "lens": s["batch"].seq_len}


# ------------------------------------------------------------------------------------------ the plain forms
def _logits(s, q, k, slope, qpos, kpos, seen):
    """Scores of q [heads, rows, 128] with k [heads, keys, 128], both 32 bits; qpos [rows], kpos [heads or 1, keys];
    `seen` [rows, keys] or None; -inf where a key is not seen."""
    z = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(D)
    if s["case"]["cap"]:
        z = s["case"]["cap"] * torch.tanh(z / s["case"]["cap"])
    if slope is not None:
        z = z - slope[:, :, None] * (qpos[None, :, None] - kpos[:, None, :]).abs()
    return z if seen is None else z.masked_fill(~seen, -math.inf)


def _softmax(z):
    """Weights and logarithms of their sums; rows that see nothing have no weight."""
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top.masked_fill(top == -math.inf, 0.0))
    total = e.sum(-1, keepdim=True)
    return e / total.masked_fill(total == 0, 1.0), (torch.log(total) + top)[..., 0]


def _grouped(x, hkv):
    """[rows][hq][...] as [hkv][group * rows][...]: the rows of one query head after another."""
    return x.unflatten(1, (hkv, -1)).transpose(0, 1).transpose(1, 2).flatten(1, 2)


def _every_query(s):
    """Plain attention of every sequence's queries, in pieces of rows that fit: (out, lse, weights' sums over the
    last `window` queries) of each sequence, heads first."""
    case, got, at, qat = s["case"], [], 0, 0
    hq, hkv = case["hq"], case["hkv"]
    G = hq // hkv
    for b, (n, m) in enumerate(zip(s["lens"], s["new"])):
        k, v = (x[:, at:at + n].float() for x in (s["K"], s["V"]))
        kpos = torch.arange(n, device=DEV)
        docs = None if s["documents"] is None else s["documents"][at:at + n]
        out, lse, sums = [], [], torch.zeros(hkv, n, device=DEV)
        step = max(1, 2 ** 29 // (hq * n))
        for i in range(0, m, step):
            j = min(m, i + step)
            qpos = torch.arange(n - m + i, n - m + j, device=DEV)
            seen = qpos[:, None] >= kpos[None, :]
            if s["prefix_len"] is not None:
                seen = seen | (kpos < s["prefix_len"][b])[None, :]
            if docs is not None:
                seen = seen & (docs[n - m + i:n - m + j, None] == docs[None, :])
            slope = None if s["slopes"] is None else s["slopes"].view(hkv, G, 1).expand(hkv, G, j - i).flatten(1)
            z = _logits(s, _grouped(s["q"][qat + i:qat + j].float(), hkv), k, slope, qpos.repeat(G), kpos[None],
                        seen.repeat(G, 1))
            if case["op"] == "weights" and "lse" in s:
                given = _grouped(s["lse"].T[qat + i:qat + j, :, None], hkv)
                last = (torch.arange(i, j, device=DEV) >= m - (case["window"] or m)).repeat(G)[None, :, None]
                sums += (torch.exp(z - given.masked_fill(given == -math.inf, 0.0)) * last).sum(1)
                continue
            p, l = _softmax(z)
            lse.append(l.unflatten(1, (G, j - i)).flatten(0, 1))
            if case["op"] == "prompt":
                out.append(torch.matmul(p, v).unflatten(1, (G, j - i)).flatten(0, 1).transpose(0, 1))
        got.append((torch.cat(out) if out else None, torch.cat(lse, 1) if lse else None, sums))
        at, qat = at + n, qat + m
    return got


def _from_pages(s, pages, table, lens):
    return torch.cat([pages[t.long()].transpose(0, 1).flatten(1, 2)[:, :n] for t, n in zip(table, lens)], 1)


def _plain_prompt(s):
    if s["case"]["page"]:
        s = dict(s, K=_from_pages(s, s["Kpg"], s["table"], s["lens"]), V=_from_pages(s, s["Vpg"], s["table"], s["lens"]))
    got = _every_query(s)
    return {"out": torch.cat([x[0] for x in got]).to(torch.bfloat16), "lse": torch.cat([x[1] for x in got], 1)}


def _plain_weights(s):
    s["sums"] += torch.cat([x[2] for x in _every_query(s)], 1)
    return {"sums": s["sums"]}


def _one_token(s, q, k, v, slopes, qpos, kpos, seen):
    """out [hq][128], lse [hq], weights per row summed over a group's heads [hkv][n]."""
    hkv = s["case"]["hkv"]
    slope = None if slopes is None else slopes.view(hkv, -1)
    z = _logits(s, q.float().view(hkv, -1, D), k.float(), slope, qpos, kpos, seen)
    p, lse = _softmax(z)
    return torch.matmul(p, v.float()).flatten(0, 1), lse.flatten(), p.sum(1)


def _plain_decode(s):
    case, at, outs, lses = s["case"], 0, [], []
    if case["page"]:
        s = dict(s, K=_from_pages(s, s["Kpg"], s["table"], s["lens"]), V=_from_pages(s, s["Vpg"], s["table"], s["lens"]))
    for b, n in enumerate(s["lens"]):
        r = slice(at, at + n)
        kpos = torch.arange(n, device=DEV)[None] if s["positions"] is None else s["positions"][:, r]
        qpos = torch.full((1,), n - 1, device=DEV) if s["q_pos"] is None else s["q_pos"][b:b + 1]
        seen = None if s["documents"] is None else (s["documents"][r] == s["q_documents"][b])[None]
        out, lse, w = _one_token(s, s["q"][b], s["K"][:, r], s["V"][:, r], s["slopes"], qpos, kpos, seen)
        if case["add"]:
            s["sums"][:, r] += w
        outs.append(out)
        lses.append(lse)
        at += n
    got = {"out": torch.stack(outs), "lse": torch.stack(lses)}
    return dict(got, sums=s["sums"]) if case["add"] else got


def _plain_shared(s):
    if s["case"]["page"]:
        s = dict(s, K=_from_pages(s, s["Kpg"], s["table"], s["lens"]), V=_from_pages(s, s["Vpg"], s["table"], s["lens"]),
                 Kp=_from_pages(s, s["Kppg"], s["ptable"], s["prefixes"]),
                 Vp=_from_pages(s, s["Vppg"], s["ptable"], s["prefixes"]))
    ends, at, outs, lses = np.cumsum([0] + s["prefixes"]), 0, [], []
    for b, n in enumerate(s["lens"]):
        i = s["of"][b]
        p = slice(int(ends[i]), int(ends[i + 1])) if i >= 0 else slice(0, 0)
        k, v = (torch.cat([x[:, p], y[:, at:at + n]], 1) for x, y in ((s["Kp"], s["K"]), (s["Vp"], s["V"])))
        kpos = torch.arange(k.shape[1], device=DEV)
        out, lse, _ = _one_token(s, s["q"][b], k, v, s["slopes"], kpos[-1:], kpos[None], None)
        outs.append(out)
        lses.append(lse)
        at += n
    return {"out": torch.stack(outs), "lse": torch.stack(lses)}


def _ranking(weights, positions, newest, recent):
    """Rows of one sequence, per head, from the first to keep to the last: recent ones by position, then by weight, ties by row."""
    fresh = positions > newest - recent
    by_weight = torch.sort(weights, dim=1, descending=True, stable=True).indices
    first = torch.where(fresh, positions, -1).gather(1, by_weight)
    return by_weight.gather(1, torch.sort(first, dim=1, descending=True, stable=True).indices)


def _plain_evict(s):
    at, to = 0, 0
    for b, (n, kept) in enumerate(zip(s["lens"], s["kept"])):
        w, pos = s["weights"][:, at:at + n], s["positions"][:, at:at + n]
        rows = torch.sort(_ranking(w, pos, s["newest"][b], s["case"]["recent"])[:, :kept], dim=1).values
        for name in ("K", "V"):
            s[name + "_out"][:, to:to + kept] = s[name][:, at:at + n].gather(1, rows[:, :, None].expand(-1, -1, D))
        s["weights_out"][:, to:to + kept] = w.gather(1, rows)
        s["positions_out"][:, to:to + kept] = pos.gather(1, rows)
        at, to = at + n, to + kept
    lens = torch.minimum(s["seq_len"], s["keep"])
    return {"K": s["K_out"], "V": s["V_out"], "weights": s["weights_out"], "positions": s["positions_out"], "lens": lens}


def _plain_insert(s):
    case, at, rows = s["case"], 0, []
    heads = torch.arange(case["hkv"], device=DEV)
    for b, n in enumerate(s["lens"]):  # (every cache is full)
        row = _ranking(s["weights"][:, at:at + n], s["positions"][:, at:at + n], s["newest"][b], case["recent"])[:, -1]
        s["K"][heads, at + row] = s["k"][b]
        s["V"][heads, at + row] = s["v"][b]
        s["weights"][heads, at + row] = 0.0
        s["positions"][heads, at + row] = s["newest"][b]
        rows.append(row.to(torch.int32))
        at += n
    return {"row": torch.stack(rows), "K": s["K"], "V": s["V"], "weights": s["weights"], "positions": s["positions"],
            "lens": s["seq_len"]}


# ------------------------------------------------------------------------------------------ what a call cannot do without
def _pairs(case):
    """Visible (query, key) pairs of one query head, for each sequence."""
    got = []
    for n, m in zip(_ints(case["lens"]), _ints(case["new"])):
        if case["docs"]:
            d = _documents(n, case["docs"])
            first = np.searchsorted(d, d[n - m:], side="left")
            got.append(int((np.arange(n - m, n) + 1 - first).sum()))
        else:
            got.append(m * (n - m) + m * (m + 1) // 2)
            if case["prefix"]:
                p = _prefix_len(m)
                got[-1] += p * (p - 1) // 2
    return got


def work(case):
    lens, hq, hkv, row = _ints(case["lens"]), case["hq"], case["hkv"], 2 * D
    if case["op"] == "prompt":
        q = sum(_ints(case["new"])) * hq
        seen = sum(lens) if not case["docs"] else sum(min(n, m + 2 * case["docs"]) for n, m in zip(lens, _ints(case["new"])))
        return {"bytes": seen * hkv * 2 * row + q * (2 * row + 4), "flops": 4.0 * D * hq * sum(_pairs(case))}
    if case["op"] == "decode":
        seen = sum(lens) if not case["docs"] else sum(min(n, case["docs"]) for n in lens)
        more = (8 if case["add"] else 0) + (4 if case["evicted"] else 0)
        return {"bytes": seen * hkv * (2 * row + more) + len(lens) * hq * (row + 4 * D + 4), "flops": 4.0 * D * hq * seen}
    if case["op"] == "shared":
        pre, of = _ints(case["prefixes"]), _ints(case["of"])
        keys = sum(lens) + sum(pre[i] for i in of if i >= 0)
        once = sum(lens) + sum(p for i, p in enumerate(pre) if i in of)
        return {"bytes": once * hkv * 2 * row + len(lens) * hq * (row + 4 * D + 4), "flops": 4.0 * D * hq * keys}
    if case["op"] == "weights":
        new = [min(m, case["window"] or m) for m in _ints(case["new"])]
        pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))
        return {"bytes": sum(lens) * hkv * (row + 8) + sum(new) * hq * (row + 4), "flops": 2.0 * D * hq * pairs}
    if case["op"] == "evict":
        kept = sum(min(n, k) for n, k in zip(lens, _ints(case["keep"])))
        return {"bytes": hkv * (sum(lens) * 8 + kept * (4 * row + 8)), "flops": float(hkv * sum(lens))}
    return {"bytes": hkv * (sum(lens) * 8 + len(lens) * (4 * row + 8)), "flops": float(hkv * sum(lens))}


# ------------------------------------------------------------------------------------------ the same in 64 bits
def _exact_head(case, q, k, v, slope, qpos, kpos, seen):
    """Attention of rows q [m][128] of one query head in 64 bits: out, lse, weights [m][n]."""
    x = q.double() @ k.double().T * D ** -0.5
    if case["cap"]:
        x = torch.tanh(x / case["cap"]) * case["cap"]
    if slope is not None:
        x -= slope.double() * (qpos[:, None] - kpos[None, :]).abs().double()
    x[~seen] = -math.inf
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    p[lse == -math.inf] = 0.0
    return (p @ v.double() if v is not None else None), lse, p


def exact(case, seed):
    s = _inputs(case, seed)
    lens, hq, hkv = s["lens"], case["hq"], case["hkv"]
    G, starts = hq // hkv, np.cumsum([0] + s["lens"])
    if case["op"] in ("evict", "insert"):
        return _exact_rows(case, s)
    if case["op"] in ("prompt", "weights"):
        qs = np.cumsum([0] + s["new"])
        out = torch.zeros(int(qs[-1]), hq, D, dtype=torch.float64, device=DEV)
        lse = torch.zeros(hq, int(qs[-1]), dtype=torch.float64, device=DEV)
        sums = s["sums"].double() if case["op"] == "weights" else None
        for b, n in enumerate(lens):
            m, a = s["new"][b], int(starts[b])
            for h in range(hq):
                k, v = s["K"][h // G, a:a + n], s["V"][h // G, a:a + n]
                kpos = torch.arange(n, device=DEV)
                for i in range(0, m, 4096):
                    rows = slice(int(qs[b]) + i, int(qs[b]) + min(m, i + 4096))
                    qpos = torch.arange(rows.start, rows.stop, device=DEV) - int(qs[b]) + n - m
                    seen = kpos[None, :] <= qpos[:, None]
                    if s["prefix_len"] is not None:
                        seen |= (kpos < int(s["prefix_len"][b]))[None, :]
                    if s["documents"] is not None:
                        d = s["documents"][a:a + n]
                        seen &= d[qpos][:, None] == d[None, :]
                    o, l, p = _exact_head(case, s["q"][rows, h], k, None if sums is not None else v,
                                          None if s["slopes"] is None else s["slopes"][h], qpos, kpos, seen)
                    if sums is None:
                        out[rows, h], lse[h, rows] = o, l
                    else:  # against the given sums of exponentials
                        p = p * torch.exp(l - s["lse"][h, rows].double())[:, None]
                        p[qpos < n - min(m, case["window"] or m)] = 0.0
                        sums[h // G, a:a + n] += p.sum(0)
        return {"out": out, "lse": lse} if sums is None else {"sums": sums}
    B = len(lens)
    out = torch.zeros(B, hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, hq, dtype=torch.float64, device=DEV)
    sums = s["sums"].double() if s.get("sums") is not None else None
    ends = np.cumsum([0] + s.get("prefixes", []))
    for b, n in enumerate(lens):
        a = int(starts[b])
        for h in range(hq):
            g = h // G
            k, v = s["K"][g, a:a + n], s["V"][g, a:a + n]
            if case["op"] == "shared" and s["of"][b] >= 0:
                p0, p1 = int(ends[s["of"][b]]), int(ends[s["of"][b] + 1])
                k, v = torch.cat([s["Kp"][g, p0:p1], k]), torch.cat([s["Vp"][g, p0:p1], v])
            kpos = torch.arange(len(k), device=DEV)
            qpos = kpos[-1:]
            if case["op"] == "decode" and s["positions"] is not None:
                kpos, qpos = s["positions"][g, a:a + n], s["q_pos"][b:b + 1]
            seen = torch.ones(1, len(k), dtype=torch.bool, device=DEV)
            if case["op"] == "decode" and s["documents"] is not None:
                seen[0] = s["documents"][a:a + n] == s["q_documents"][b]
            o, l, p = _exact_head(case, s["q"][b, h:h + 1], k, v, None if s["slopes"] is None else s["slopes"][h],
                                  qpos, kpos, seen)
            out[b, h], lse[b, h] = o[0], l[0]
            if sums is not None:
                sums[g, a:a + n] += p[0]
    return {"out": out, "lse": lse} if sums is None else {"out": out, "lse": lse, "sums": sums}


def _exact_rows(case, s):
    """Eviction and insertion, ranked on the host by (recent, position, weight, row)."""
    lens, hkv = s["lens"], case["hkv"]
    w, pos, newest = s["weights"].cpu().numpy(), s["positions"].cpu().numpy(), s["newest"].cpu().numpy()
    starts, picked, victims = np.cumsum([0] + lens), [[] for _ in range(hkv)], np.zeros((len(lens), hkv), np.int64)
    for b, n in enumerate(lens):
        a = int(starts[b])
        for g in range(hkv):
            fresh = pos[g, a:a + n] > newest[b] - case["recent"]
            order = np.lexsort((np.arange(n), np.where(fresh, 0.0, -w[g, a:a + n]), np.where(fresh, -pos[g, a:a + n], 1)))
            victims[b, g] = order[-1]
            if case["op"] == "evict":
                picked[g].append(a + np.sort(order[:_ints(case["keep"])[b]]))
    if case["op"] == "evict":
        rows = torch.as_tensor(np.stack([np.concatenate(x) for x in picked]), device=DEV)
        K, V = (s[x].double().gather(1, rows[:, :, None].expand(-1, -1, D)) for x in ("K", "V"))
        return {"K": K, "V": V, "weights": s["weights"].double().gather(1, rows), "positions": None, "lens": None}
    K, V, sums = s["K"].double(), s["V"].double(), s["weights"].double()
    for b, g in np.ndindex(len(lens), hkv):
        at = int(starts[b]) + int(victims[b, g])
        K[g, at], V[g, at], sums[g, at] = s["k"][b, g].double(), s["v"][b, g].double(), 0.0
    return {"row": None, "K": K, "V": V, "weights": sums, "positions": None, "lens": None}
