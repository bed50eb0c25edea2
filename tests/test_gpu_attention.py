"""Prompt attention, scored decode and shared prefixes against a plain 64-bit
implementation (tests/attention_ref.py), at the sizes and masks where a tile, a
split or a mask may go wrong.  Tolerances are counted roundings."""
import numpy as np
import pytest
import torch

from tests import attention_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _randn(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def _batch(lens, hq, hkv, spare=0):
    import paper_2502_12216_amd as T
    return T.RaggedBatch(lens, hq, hkv, capacities=[n + spare for n in lens] if spare else None)


def _documents(n, mean, seed=0):
    """Runs of documents, and the ids in an order that is not the positions'."""
    cuts = np.random.default_rng([n, mean, seed]).exponential(mean, size=4 * n // mean + 8).astype(np.int64).cumsum()
    ids = np.searchsorted(cuts, np.arange(n), side="right")
    return ((ids * 7919) % 1009 - 300).astype(np.int32)


def check_prompt(lens, new, hq, hkv, cap=0.0, alibi=False, docs=0, prefix=None, page=0, spare=0, seed=1, spoil=None,
                 stream=None):
    import paper_2502_12216_amd as T
    batch = _batch(lens, hq, hkv, spare)
    K, V = _randn(seed, hkv, batch.total, 128), _randn(seed + 1, hkv, batch.total, 128)
    starts = [int(x) for x in batch.kv_indptr_host]
    if spare:  # rows behind a sequence's tokens hold anything
        for b, n in enumerate(lens):
            K[:, starts[b] + n:starts[b + 1]] = float("nan")
            V[:, starts[b] + n:starts[b + 1]] = float("nan")
    q = _randn(seed + 2, sum(new), hq, 128, scale=2.0)
    sl = R.slopes(hq) if alibi else None
    document = None
    if docs:
        document = torch.zeros(batch.total, dtype=torch.int32, device=DEV)
        for b, n in enumerate(lens):
            document[starts[b]:starts[b] + n] = torch.as_tensor(_documents(n, docs, seed), device=DEV)
    pre = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=DEV)
    if spoil:
        spoil(K, V)
    mod = T.ScoreMod(cap=cap, slopes=sl, documents=document, prefix_len=pre)
    att = T.PromptAttention(batch, new)
    att.out.fill_(float("nan"))
    att.lse.fill_(float("nan"))
    if page:
        assert not spare
        Kp, table = R.pages(K, lens, page, seed)
        Vp, _ = R.pages(V, lens, page, seed)
        out, lse = att.paged(q, T.PagedCache(Kp, Vp, table), mod, stream=stream)
    else:
        out, lse = att(q, K, V, mod, stream=stream)
    torch.cuda.synchronize()
    G, at, worst = hq // hkv, 0, 0.0
    for b, (n, m) in enumerate(zip(lens, new)):
        kpos, qpos = torch.arange(n, device=DEV), torch.arange(n - m, n, device=DEV)
        seen = (kpos[None, :] <= qpos[:, None]) if pre is None else \
            (kpos[None, :] <= qpos[:, None]) | ((kpos < pre[b])[None, :] & (qpos >= 0)[:, None])
        if document is not None:
            d = document[starts[b]:starts[b] + n]
            seen = seen & (d[qpos.clamp_min(0)][:, None] == d[None, :]) if n else seen
        for h in range(hq):
            g = h // G
            o, l, _, ma, off = R.attend(q[at:at + m, h], K[g, starts[b]:starts[b] + n], V[g, starts[b]:starts[b] + n], qpos,
                                        kpos, seen, cap, float(sl[h]) if alibi else 0.0)
            worst = max(worst, R.close(out[at:at + m, h], o, R.tolerance_bf16(ma, off, o), f"out b={b} h={h}"))
            R.close(lse[h, at:at + m], l, R.tolerance_lse(off, l), f"lse b={b} h={h}")
        at += m
    return att, q, K, V, mod, out, lse, worst


@pytest.mark.parametrize("lens,new,hq,hkv", [
    ([1], [1], 8, 2),                           # one token
    ([33], [33], 8, 8),                         # one head per KV head: 64-row tiles
    ([5, 0, 130, 1], [5, 0, 130, 1], 4, 2),     # a sequence without tokens, 256-row tiles
    ([97, 70], [97, 7], 16, 2),                 # eight heads per KV head
    ([300, 1000], [9, 2], 8, 2),                # chunks: 64-row tiles, keys split among waves and workgroups
    ([4100], [3], 8, 2),                        # a few tokens against a long cache: 32-row tiles, splits
    ([2500, 64], [30, 30], 8, 2),               # 128-row tiles
    ([700, 64, 257], [700, 64, 200], 2, 1),
    ([0], [0], 8, 2),
    ([3, 0, 40], [5, 2, 41], 8, 2),             # more queries than tokens: the first ones see nothing
])
def test_prompt_causal(lens, new, hq, hkv):
    check_prompt(lens, new, hq, hkv)


@pytest.mark.parametrize("kw", [
    dict(cap=30.0), dict(cap=0.5), dict(alibi=True), dict(cap=50.0, alibi=True), dict(docs=40), dict(docs=5, cap=20.0),
    dict(prefix=[100, 0, 5000]), dict(prefix=[1, 300, 17], alibi=True, docs=200), dict(page=16), dict(page=7, docs=90),
    dict(spare=37), dict(spare=5, prefix=[500, 2, 64], cap=40.0),
])
@pytest.mark.parametrize("new", [[411, 260, 64], [8, 1, 2], [30, 3, 17], [16, 9, 64]])
def test_prompt_scores_and_masks(kw, new):
    check_prompt([411, 260, 1064], new, 8, 2, **kw)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new", [[200], [5], [20]])
def test_prompt_masked_places_may_hold_anything(value, new):
    """Keys and values that a query does not see (a later token, another document) are not finite; queries
    that see them have the formula's result."""
    def spoil(K, V):
        K[0, 197, 3] = value
        V[0, 190, 5:9] = value
        V[1, 198] = value
        V[0, 150, 1] = value
    check_prompt([200], new, 4, 2, docs=30, spoil=spoil)


def test_prompt_large_scores():
    """Scores far beyond the exponential's range: the running maximum carries them."""
    check_prompt([300], [300], 4, 2, seed=5, spoil=lambda K, V: K.mul_(64.0))


def check_decode(lens, hq, hkv, cap=0.0, alibi=False, docs=0, page=0, positions=False, add=False, spare=0, seed=3,
                 spoil=None, missing=False, stream=None):
    import paper_2502_12216_amd as T
    batch = _batch(lens, hq, hkv, spare)
    B, G = len(lens), hq // hkv
    K, V = _randn(seed, hkv, batch.total, 128), _randn(seed + 1, hkv, batch.total, 128)
    q = _randn(seed + 2, B, hq, 128, scale=2.0)
    starts = [int(x) for x in batch.kv_indptr_host]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    pos = qp = document = qd = sums = None
    if positions:
        pos = torch.randperm(hkv * batch.total, generator=g, device=DEV).to(torch.int32).view(hkv, batch.total)
        qp = torch.tensor([hkv * batch.total + 3 * b for b in range(B)], dtype=torch.int32, device=DEV)
    if docs:
        document = torch.zeros(batch.total, dtype=torch.int32, device=DEV)
        for b, n in enumerate(lens):
            document[starts[b]:starts[b] + n] = torch.as_tensor(_documents(n, docs, seed), device=DEV)
        qd = torch.stack([document[starts[b] + n // 2] if n else document.new_zeros(()) for b, n in enumerate(lens)]).contiguous()
        if missing:
            qd[0] = 10 ** 6  # a document that no row belongs to
    if spoil:
        spoil(K, V, document, qd)
    if add:
        sums = torch.rand(hkv, batch.total, generator=g, device=DEV)
        before = sums.clone()
    mod = T.ScoreMod(cap=cap, slopes=R.slopes(hq) if alibi else None, documents=document)
    dec = T.ScoredDecoder(batch)
    dec.out.fill_(float("nan"))
    dec.lse.fill_(float("nan"))
    kw = dict(positions=pos, q_pos=qp, q_documents=qd, weights=sums, stream=stream)
    if page:
        Kp, table = R.pages(K, lens, page, seed)
        Vp, _ = R.pages(V, lens, page, seed)
        out, lse = dec.paged(q, T.PagedCache(Kp, Vp, table), mod, **kw)
    else:
        out, lse = dec(q, K, V, mod, **kw)
    torch.cuda.synchronize()
    if add:
        added = torch.zeros_like(sums, dtype=torch.float64)
        slack = torch.zeros_like(added)
    for b, n in enumerate(lens):
        r = slice(starts[b], starts[b] + n)
        for h in range(hq):
            kv = h // G
            kpos = torch.arange(n, device=DEV) if pos is None else pos[kv, r]
            qpos = torch.tensor([n - 1], device=DEV) if qp is None else qp[b:b + 1]
            seen = torch.ones(1, n, dtype=torch.bool, device=DEV)
            if document is not None:
                seen = (document[r] == qd[b])[None]
            o, l, p, ma, off = R.attend(q[b, h:h + 1], K[kv, r], V[kv, r], qpos, kpos, seen, cap,
                                        float(R.slopes(hq)[h]) if alibi else 0.0)
            R.close(out[b, h:h + 1], o, R.tolerance_fp32(ma, off, o), f"out b={b} h={h}")
            R.close(lse[b, h:h + 1], l, R.tolerance_lse(off, l), f"lse b={b} h={h}")
            if add:
                added[kv, r] += p[0]
                slack[kv, r] += p[0] * (2.1 * off[0] + 64 * 2.0 ** -24)
    if add:  # rows behind a sequence's tokens keep their sums
        ref = before.double() + added
        R.close(sums, ref, slack + 2.0 ** -23 * ref.abs(), "sums")
    return out


@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("kw", [
    dict(), dict(cap=30.0), dict(alibi=True, cap=50.0, add=True), dict(docs=50, add=True), dict(page=16, alibi=True),
    dict(page=5, docs=100, add=True), dict(positions=True, alibi=True, add=True), dict(spare=9, add=True),
    dict(docs=20, missing=True, alibi=True, positions=True, add=True),
])
def test_scored_decode(hq, hkv, kw):
    check_decode([700, 1, 0, 2049], hq, hkv, **kw)


@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (16, 2)])
def test_scored_decode_many_workgroups(hq, hkv):
    check_decode([33000, 20011, 5], hq, hkv, cap=50.0, alibi=True, add=True)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (16, 2)])
def test_scored_decode_masked_places_may_hold_anything(value, hq, hkv):
    def spoil(K, V, document, qd):
        other = torch.nonzero(document[:500] != qd[0])[:, 0]
        K[:, other[::3]] = value
        V[:, other[1::3]] = value
    check_decode([500], hq, hkv, docs=60, spoil=spoil, add=True)


def test_scored_decode_equals_dense_decode_bit_for_bit_without_a_rule():
    """Without a cap, bias or documents the sums are those of the dense decode."""
    import paper_2502_12216_amd as T
    batch = _batch([3001, 17, 900], 8, 2)
    K, V, q = _randn(1, 2, batch.total, 128), _randn(2, 2, batch.total, 128), _randn(3, 3, 8, 128)
    a = T.DenseDecoder(batch)(q, K, V)
    b, _ = T.ScoredDecoder(batch)(q, K, V)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def check_shared(prefixes, of, lens, hq, hkv, cap=0.0, alibi=False, page=0, spare=0, seed=4):
    import paper_2502_12216_amd as T
    batch = _batch(lens, hq, hkv, spare)
    B, G = len(lens), hq // hkv
    K, V = _randn(seed, hkv, batch.total, 128), _randn(seed + 1, hkv, batch.total, 128)
    Kp, Vp = _randn(seed + 3, hkv, sum(prefixes), 128), _randn(seed + 4, hkv, sum(prefixes), 128)
    q = _randn(seed + 2, B, hq, 128, scale=2.0)
    starts, ends = [int(x) for x in batch.kv_indptr_host], np.cumsum([0] + list(prefixes))
    mod = T.ScoreMod(cap=cap, slopes=R.slopes(hq) if alibi else None)
    dec = T.SharedPrefixDecoder(batch, prefixes, of)
    dec.workspace.fill_(255)  # NaN everywhere: contents on entry are irrelevant
    if page:
        caches = []
        for x, y, n in ((Kp, Vp, prefixes), (K, V, lens)):
            a, table = R.pages(x, n, page, seed)
            caches.append(T.PagedCache(a, R.pages(y, n, page, seed)[0], table))
        out, lse = dec.paged(q, *caches, mod)
    else:
        out, lse = dec(q, Kp, Vp, K, V, mod)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        p0, p1 = (int(ends[of[b]]), int(ends[of[b] + 1])) if of[b] >= 0 else (0, 0)
        for h in range(hq):
            g = h // G
            k, v = (torch.cat([x[g, p0:p1], y[g, starts[b]:starts[b] + n]]) for x, y in ((Kp, K), (Vp, V)))
            kpos = torch.arange(len(k), device=DEV)
            seen = torch.ones(1, len(k), dtype=torch.bool, device=DEV)
            o, l, _, ma, off = R.attend(q[b, h:h + 1], k, v, torch.tensor([len(k) - 1], device=DEV), kpos, seen, cap,
                                        float(R.slopes(hq)[h]) if alibi else 0.0)
            R.close(out[b, h:h + 1], o, R.tolerance_fp32(ma, off, o), f"out b={b} h={h}")
            R.close(lse[b, h:h + 1], l, R.tolerance_lse(off, l), f"lse b={b} h={h}")


@pytest.mark.parametrize("prefixes,of,lens,hq,hkv", [
    ([1000], [0] * 4, [3, 9, 0, 40], 8, 2),                       # 16 rows: one wave per tile of keys
    ([4097], [0] * 12, list(range(12)), 8, 2),                    # 48 rows
    ([777], [0] * 27, [5] * 27, 8, 2),                            # 108 rows
    ([300], [0] * 70, [2] * 70, 8, 2),                            # two row tiles
    ([64, 0, 1500, 31], [2, 0, -1, 2, 1, 3, 3, 2, -1], [7, 100, 50, 0, 0, 1, 2, 600, 0], 4, 4),
    ([500, 900], [1, 1, 0, 1, 1], [30, 2, 5, 1, 300], 16, 2),
    ([900], [0], [0], 8, 1),
    ([10], [-1, -1], [5, 0], 8, 2),                               # nobody has a prefix, one has nothing at all
])
@pytest.mark.parametrize("kw", [dict(), dict(cap=30.0, alibi=True), dict(page=16), dict(page=9, alibi=True), dict(spare=11)])
def test_shared_prefix(prefixes, of, lens, hq, hkv, kw):
    check_shared(prefixes, of, lens, hq, hkv, **kw)


def test_calls_on_another_stream_and_twice_give_the_same():
    """Work enqueued on a side stream, and results that do not depend on scheduling."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    check_prompt([900], [900], 8, 2, cap=30.0, stream=side)
    check_decode([5000, 3], 8, 2, alibi=True, add=True, stream=side)
    att, q, K, V, mod, out, lse, _ = check_prompt([5000], [40], 8, 2, alibi=True)
    first = out.clone()
    for _ in range(3):
        again, _ = att(q, K, V, mod)
        assert torch.equal(again, first)
