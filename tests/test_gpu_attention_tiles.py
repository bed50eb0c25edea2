"""Prompt and shared-prefix attention at sizes where the row tile and the splits of
the keys differ (the small shapes of test_gpu_attention.py all take 32 rows to a
tile), tiles that hold nothing finite, and caps of every degree of the polynomial."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attention import DEV, _batch, _randn, check_decode, check_prompt
from tests.test_gpu_evict import check_weights

pytestmark = pytest.mark.gpu

TILES = [
    ([400, 333, 397], [300, 290, 299], 32, 8),        # 64 rows
    ([700, 650, 31], [700, 650, 31], 12, 6),
    ([400, 390, 131, 400], [200, 200, 131, 199], 32, 8),  # 128 rows
    ([4000], [300], 16, 2),                           # and splits
    ([400, 1, 0, 399, 400, 380], [200, 1, 0, 200, 200, 199], 32, 8),  # 256 rows
    ([400] * 6, [200] * 6, 32, 8),
    ([2100, 1900], [700, 650], 12, 6),                # and splits
]


@pytest.mark.parametrize("lens,new,hq,hkv", TILES)
@pytest.mark.parametrize("kw", [dict(), dict(cap=30.0, page=16), dict(alibi=True, prefix=100, spare=3), dict(docs=60),
                                dict(docs=300, page=7, alibi=True, cap=3.0)])
def test_prompt_row_tiles(lens, new, hq, hkv, kw):
    if "prefix" in kw:
        kw = dict(kw, prefix=[kw["prefix"] + 37 * b for b in range(len(lens))])
    check_prompt(lens, new, hq, hkv, **kw)


@pytest.mark.parametrize("lens,new,hq,hkv", [([400, 333], [300, 290], 32, 8), ([400, 390, 131, 400], [200, 200, 131, 199], 32, 8),
                                             ([400] * 6, [200] * 6, 32, 8), ([900, 700], [300, 260], 12, 6)])
def test_prompt_row_tiles_with_values_that_are_not_finite(lens, new, hq, hkv):
    def spoil(K, V):
        for i, value in enumerate((float("nan"), float("inf"), -float("inf"))):
            V[i::3, 211 + i, 5 * i:5 * i + 2] = value
            V[0, 350 + 3 * i] = value
            K[1, 300 + 7 * i, 3] = value
    check_prompt(lens, new, hq, hkv, docs=25, spoil=spoil)


@pytest.mark.parametrize("lens,new,hq,hkv,docs", [
    ([120] * 60, [120] * 60, 32, 8, 30), ([3400, 3, 2900], [3400, 3, 2900], 32, 8, 300), ([40, 0] * 40, [42, 1] * 40, 32, 8, 20),
])
@pytest.mark.parametrize("kw", [dict(), dict(prefix=True, page=16), dict(spare=3, alibi=True, cap=9.0)])
def test_prompt_of_many_documents(lens, new, hq, hkv, docs, kw):
    """Enough row tiles that the long ones are started first."""
    if "prefix" in kw:
        kw = dict(kw, prefix=[(37 * b) % 200 for b in range(len(lens))])
    check_prompt(lens, new, hq, hkv, docs=docs, **kw)


@pytest.mark.parametrize("new", [200, 64, 5, 1])
@pytest.mark.parametrize("rows", [slice(0, 1), slice(0, 64), slice(64, 128), slice(96, 128), slice(0, 200)])
def test_prompt_tiles_of_nan_keys(new, rows):
    """Every score of a tile, a wave's keys or a split is NaN: so is the row that sees one of them."""
    def spoil(K, V):
        K[:, rows] = float("nan")
    check_prompt([200], [new], 4, 2, spoil=spoil)


def test_prompt_documents_of_one_nan_key():
    def spoil(K, V):
        K[:, 3:400:5] = float("nan")
    check_prompt([400], [400], 4, 2, docs=2, spoil=spoil)


@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("rows", [slice(0, 1), slice(0, 4), slice(64, 128), slice(3, 4)])
def test_decode_groups_of_nan_keys(hq, hkv, rows):
    def spoil(K, V, document, qd):
        K[0, rows] = float("nan")
    check_decode([333, 1, 50], hq, hkv, spoil=spoil)
    check_decode([4], hq, hkv, spoil=spoil, add=True)


@pytest.mark.parametrize("scale", [0.3, 1.0, 8.0])
def test_caps_of_every_size(scale):
    """Scores that stay within 0.375 of the cap, within 0.75, and beyond; and all in one prompt."""
    def spoil(K, V):
        K.mul_(scale)
        K[:, 300:] *= 4
    for cap in (2.0, 20.0, 200.0):
        check_prompt([500], [500], 4, 2, cap=cap, spoil=spoil)
    check_prompt([400, 390, 131, 400], [200, 200, 131, 199], 32, 8, cap=20.0, spoil=spoil)
    check_decode([500], 8, 2, cap=20.0, spoil=lambda K, V, d, q: spoil(K, V))


@pytest.mark.parametrize("cap", [0.7, 6.0, 30.0])
@pytest.mark.parametrize("docs", [0, 40])
def test_weights_of_capped_prompts(cap, docs):
    check_weights([700, 300], [700, 300], 8, 2, 0, cap=cap, docs=docs)


@pytest.mark.parametrize("prefix,members,hq,hkv", [
    (100, 512, 32, 8),   # 64 rows, one split
    (1000, 150, 32, 8),  # and splits
    (300, 512, 64, 8),   # 128 rows, one split
    (1000, 200, 32, 8),  # and splits
    (100, 512, 64, 8),   # 256 rows
])
@pytest.mark.parametrize("kw", [dict(), dict(cap=20.0), dict(page=16, alibi=True)])
def test_shared_prefix_row_tiles(prefix, members, hq, hkv, kw):
    """Many sequences of one prefix, a head at a time: own tokens are keys that one row sees."""
    import paper_2502_12216_amd as T
    lens = [i % 4 for i in range(members)]
    batch = _batch(lens, hq, hkv)
    K, V = _randn(1, hkv, batch.total, 128), _randn(2, hkv, batch.total, 128)
    Kp, Vp, q = _randn(3, hkv, prefix, 128), _randn(4, hkv, prefix, 128), _randn(5, members, hq, 128, scale=2.0)
    sl = R.slopes(hq) if "alibi" in kw else None
    mod = T.ScoreMod(cap=kw.get("cap", 0.0), slopes=sl)
    dec = T.SharedPrefixDecoder(batch, [prefix], [0] * members)
    dec.workspace.fill_(255)  # NaN everywhere: contents on entry are irrelevant
    if "page" in kw:
        caches = []
        for x, y, n in ((Kp, Vp, [prefix]), (K, V, lens)):
            a, table = R.pages(x, n, kw["page"])
            caches.append(T.PagedCache(a, R.pages(y, n, kw["page"])[0], table))
        out, lse = dec.paged(q, *caches, mod)
    else:
        out, lse = dec(q, Kp, Vp, K, V, mod)
    torch.cuda.synchronize()
    own = torch.as_tensor(lens, device=DEV)
    of = torch.repeat_interleave(torch.arange(members, device=DEV), own)
    kpos = torch.cat([torch.arange(prefix, device=DEV)] + [prefix + torch.arange(n, device=DEV) for n in lens])
    seen = torch.cat([torch.ones(members, prefix, dtype=torch.bool, device=DEV), of[None] == torch.arange(members, device=DEV)[:, None]], 1)
    for h in range(hq):
        k, v = (torch.cat([x[h * hkv // hq], y[h * hkv // hq]]) for x, y in ((Kp, K), (Vp, V)))
        o, l, _, ma, off = R.attend(q[:, h], k, v, prefix + own - 1, kpos, seen, mod.cap, float(sl[h]) if sl is not None else 0.0)
        R.close(out[:, h], o, R.tolerance_fp32(ma, off, o), f"out h={h}")
        R.close(lse[:, h], l, R.tolerance_lse(off, l), f"lse h={h}")


@pytest.mark.parametrize("rows", [slice(0, 1), slice(0, 32), slice(32, 160)])
def test_shared_prefix_of_nan_keys(rows):
    """A tile of the prefix's keys is NaN: so are its sequences, and only those."""
    import paper_2502_12216_amd as T
    batch, hq, hkv = _batch([3, 0, 9], 8, 2), 8, 2
    K, V, q = _randn(1, hkv, batch.total, 128), _randn(2, hkv, batch.total, 128), _randn(3, 3, hq, 128)
    Kp, Vp = _randn(4, hkv, 500, 128), _randn(5, hkv, 500, 128)
    Kp[0, rows] = float("nan")
    out, lse = T.SharedPrefixDecoder(batch, [500], [0, 0, -1])(q, Kp, Vp, K, V)
    torch.cuda.synchronize()
    assert torch.isnan(out[:2, :4]).all() and torch.isnan(lse[:2, :4]).all()
    assert torch.isfinite(out[:2, 4:]).all() and torch.isfinite(out[2]).all() and torch.isfinite(lse[2]).all()


def test_rows_beyond_two_to_the_31_elements():
    """A cache whose later rows start past 2^31 elements (and past 2^32 bytes): KV head 1 and the second sequence."""
    import paper_2502_12216_amd as T
    n = 9_000_000  # rows of one KV head: 2 x 9e6 x 128 elements
    lens = [300, 500]
    batch = T.RaggedBatch(lens, 8, 2, capacities=[n - 600, 600])
    K, V = (torch.zeros(2, batch.total, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    parts = []
    for b, (s, m) in enumerate(zip([0, n - 600], lens)):
        k, v = _randn(10 + b, 2, m, 128), _randn(20 + b, 2, m, 128)
        K[:, s:s + m], V[:, s:s + m] = k, v
        parts.append((k, v))
    small = T.RaggedBatch(lens, 8, 2)
    Ks, Vs = (torch.cat([p[i] for p in parts], 1).contiguous() for i in range(2))
    mod = T.ScoreMod(cap=30.0, slopes=R.slopes(8))
    q, qd = _randn(30, 200, 8, 128), _randn(31, 2, 8, 128)
    results = []
    for bt, k, v in ((batch, K, V), (small, Ks, Vs)):
        att = T.PromptAttention(bt, [120, 80])
        out, lse = att(q, k, v, mod)
        sums = torch.zeros(2, bt.total, device=DEV)
        att.add_weights(q, k, lse, sums, mod)
        o, l = T.ScoredDecoder(bt)(qd, k, v, mod, weights=sums)
        starts = [int(x) for x in bt.kv_indptr_host]
        rows = torch.cat([sums[:, s:s + m] for s, m in zip(starts, lens)], 1)
        dest = T.RaggedBatch([0, 0], 2, 2, capacities=[100, 100])
        src = T.RaggedBatch(lens, 2, 2, capacities=[n - 600, 600]) if bt is batch else T.RaggedBatch(lens, 2, 2)
        Ko, Vo = (torch.zeros(2, 200, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        wo, po = torch.zeros(2, 200, device=DEV), torch.zeros(2, 200, dtype=torch.int32, device=DEV)
        T.CacheEvictor(src, dest, 16)(k, v, sums, torch.tensor([100, 100], dtype=torch.int32, device=DEV), Ko, Vo, wo, po)
        torch.cuda.synchronize()
        results.append([x.clone() for x in (out, lse, o, l, rows, Ko, Vo, po)])
    big, ref = results
    # the same sums in possibly another order of splits: a bf16 rounding each, and 32-bit roundings
    for x, y, tol in zip(big, ref, (2.0 ** -6, 1e-4, 1e-4, 1e-4, 1e-4)):
        assert ((x.double() - y.double()).abs() <= tol * (1 + y.double().abs())).all()
    for x, y in zip(big[5:], ref[5:]):
        assert torch.equal(x, y)


def test_insert_beyond_two_to_the_31_elements():
    import paper_2502_12216_amd as T
    n = 9_000_000
    batch = T.RaggedBatch([0, 50], 2, 2, capacities=[n, 50])
    K, V = (torch.zeros(2, batch.total, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    w = torch.rand(2, batch.total, device=DEV)
    p = torch.arange(batch.total, dtype=torch.int32, device=DEV).repeat(2, 1)
    k, v = _randn(1, 2, 2, 128), _randn(2, 2, 2, 128)
    before = w.clone()
    rows = T.TokenInserter(batch, 4)(k, v, K, V, w, p, torch.tensor([0, n + 50], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for g in range(2):
        at = n + int(before[g, n:n + 47].argmin())  # (the newest three and the new one are recent)
        assert int(rows[0, g]) == 0 and int(rows[1, g]) == at - n
        assert torch.equal(K[g, 0], k[0, g]) and torch.equal(K[g, at], k[1, g]) and torch.equal(V[g, at], v[1, g])
        assert int(p[g, at]) == n + 50 and float(w[g, at]) == 0.0


@pytest.mark.parametrize("docs", [0, 70])
@pytest.mark.parametrize("window", [0, 260])
def test_weights_of_nan_rows_reach_the_keys_they_see(docs, window):
    """A query that is NaN gives NaN to the keys it sees, of its KV head, and leaves the others' sums."""
    import paper_2502_12216_amd as T
    n, hq, hkv = 300, 8, 2
    batch = _batch([n], hq, hkv)
    K, V, q = _randn(1, hkv, n, 128), _randn(2, hkv, n, 128), _randn(3, n, hq, 128)
    document = torch.arange(n, dtype=torch.int32, device=DEV) // docs if docs else None
    mod = T.ScoreMod(documents=document)
    att = T.PromptAttention(batch, [n])
    results = []
    for spoil in (False, True):
        if spoil:
            q[50, 1], q[210, 6] = float("nan"), float("nan")
        _, lse = att(q, K, V, mod)
        assert bool(torch.isnan(lse).any()) == spoil
        results.append(att.add_weights(q, K, lse, torch.zeros(hkv, n, device=DEV), mod, window=window).clone())
    torch.cuda.synchronize()
    clean, got = results
    seen = torch.zeros(hkv, n, dtype=torch.bool, device=DEV)
    for g, i in ((0, 50), (1, 210)):
        if window == 0 or i >= n - window:
            seen[g, (i // docs * docs if docs else 0):i + 1] = True
    assert torch.equal(torch.isnan(got), seen)
    assert torch.equal(got[~seen], clean[~seen])


def test_graphs_that_share_a_workspace():
    """Prompts with documents (ranges, order and splits in the workspace), weights and an eviction, captured in two
    graphs over one workspace and replayed in turn, with eager work between."""
    import paper_2502_12216_amd as T
    runs = []
    ws = None
    for lens, new, docs in (([3400, 300, 2900], [3400, 300, 2900], 250), ([20000], [64], 9000)):
        batch = _batch(lens, 32, 8)
        ws = torch.empty(2 ** 28, dtype=torch.uint8, device=DEV) if ws is None else ws
        att = T.PromptAttention(batch, new, workspace=ws)
        assert att.workspace is ws
        q, K, V = (_randn(i, n, h, 128) for i, n, h in ((1, sum(new), 32), (2, 8, batch.total), (3, 8, batch.total)))
        mod = T.ScoreMod(cap=30.0, documents=(torch.arange(batch.total, device=DEV) // docs).int())
        dest = T.RaggedBatch([0] * len(lens), 32, 8, capacities=[100] * len(lens))
        ev = T.CacheEvictor(batch, dest, 10)
        assert ws.numel() >= ev.workspace.numel()
        ev.workspace = ws
        sums, keep = torch.zeros(8, batch.total, device=DEV), torch.full((len(lens),), 100, dtype=torch.int32, device=DEV)
        outs = [torch.zeros(8, dest.total, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)] + \
            [torch.zeros(8, dest.total, device=DEV), torch.zeros(8, dest.total, dtype=torch.int32, device=DEV)]

        def step(att=att, q=q, K=K, V=V, mod=mod, ev=ev, sums=sums, keep=keep, outs=outs):
            out, lse = att(q, K, V, mod)
            sums.zero_()
            att.add_weights(q, K, lse, sums, mod, window=50)
            ev(K, V, sums, keep, *outs)
            return [out, lse, sums] + outs
        runs.append((step, q))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for step, _ in runs:
            step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for step, q in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = step()
        graphs.append((graph, kept, q, step))
    for turn in range(4):
        for i, (graph, kept, q, step) in enumerate(graphs):
            q.copy_(_randn(100 + 10 * turn + i, *q.shape))
            want = [x.clone() for x in step()]
            for x in kept:
                x.zero_()
            ws.random_(0, 255)
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(kept, want):
                assert torch.equal(x, y), (turn, i)
