"""Accumulated weights of prompts, eviction, insertion, and the cache that runs
them together, against plain 64-bit (weights) and exact (rows) references."""
import numpy as np
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attention import DEV, _documents, _randn, check_prompt

pytestmark = pytest.mark.gpu


def check_weights(lens, new, hq, hkv, window, cap=0.0, alibi=False, docs=0, prefix=None, spare=0):
    att, q, K, V, mod, out, lse, _ = check_prompt(lens, new, hq, hkv, cap=cap, alibi=alibi, docs=docs, prefix=prefix,
                                                  spare=spare)
    batch, G, at = att.batch, hq // hkv, 0
    g = torch.Generator(device=DEV)
    g.manual_seed(9)
    sums = torch.rand(hkv, batch.total, generator=g, device=DEV)
    ref, slack = sums.double(), torch.zeros(hkv, batch.total, dtype=torch.float64, device=DEV)
    got = att.add_weights(q, K, lse, sums, mod, window=window)
    assert got is sums
    torch.cuda.synchronize()
    for b, (n, m) in enumerate(zip(lens, new)):
        s0 = int(batch.kv_indptr_host[b])
        kpos, qpos = torch.arange(n, device=DEV), torch.arange(n - m, n, device=DEV)
        seen = kpos[None, :] <= qpos[:, None]
        if prefix is not None:
            seen = seen | ((kpos < prefix[b])[None, :] & (qpos >= 0)[:, None])
        if mod.documents is not None:
            d = mod.documents[s0:s0 + n]
            seen = seen & (d[qpos.clamp_min(0)][:, None] == d[None, :])
        last = (torch.arange(m, device=DEV) >= m - window) if window else torch.ones(m, dtype=torch.bool, device=DEV)
        for h in range(hq):
            _, l, p, _, off = R.attend(q[at:at + m, h], K[h // G, s0:s0 + n], V[h // G, s0:s0 + n], qpos, kpos, seen, cap,
                                       float(R.slopes(hq)[h]) if alibi else 0.0)
            # against the lse that the call was given, whose own error enters every weight
            given = lse[h, at:at + m].double()
            p = p * torch.exp(torch.where(l == -np.inf, 0.0, l - given))[:, None] * last[:, None]
            ref[h // G, s0:s0 + n] += p.sum(0)
            rounding = 2.0 ** -24 * (16 + 8 * torch.where(l == -np.inf, 0.0, l).abs())
            slack[h // G, s0:s0 + n] += (p * (1.1 * off + rounding)[:, None]).sum(0)
        at += m
    # sums in 32 bits: at most one rounding of the result per query row of a lane, and the splits
    terms = sum(new) * G / 16 + 64
    R.close(sums, ref, slack + terms * 2.0 ** -24 * ref, "sums")


@pytest.mark.parametrize("lens,new,hq,hkv,window", [
    ([1], [1], 8, 2, 0), ([300, 0, 77], [300, 0, 77], 8, 2, 0), ([700], [700], 4, 4, 0), ([513, 256], [513, 256], 16, 2, 10),
    ([4000, 257], [40, 3], 8, 2, 0), ([4000, 300], [64, 64], 8, 2, 16), ([2000], [2000], 2, 1, 0),
    ([3, 40], [5, 41], 8, 2, 0),
])
def test_prompt_weights(lens, new, hq, hkv, window):
    check_weights(lens, new, hq, hkv, window)


@pytest.mark.parametrize("kw", [dict(cap=30.0), dict(alibi=True), dict(docs=60, cap=20.0), dict(prefix=[50, 400]),
                                dict(prefix=[300, 5], docs=100, alibi=True), dict(spare=50)])
@pytest.mark.parametrize("window", [0, 33])
def test_prompt_weights_scores_and_masks(kw, window):
    check_weights([411, 700], [411, 300], 8, 2, window, **kw)


def _cache_inputs(lens, hkv, seed, spare=0, values="pareto"):
    import paper_2502_12216_amd as T
    batch = T.RaggedBatch(lens, hkv, hkv, capacities=[n + spare for n in lens] if spare else None)
    K, V = _randn(seed, hkv, batch.total, 128), _randn(seed + 1, hkv, batch.total, 128)
    rng = np.random.default_rng(seed)
    if values == "pareto":
        w = rng.random((hkv, batch.total)) ** -0.7 - 1
        w[rng.random(w.shape) < 0.2] = 0.0
    elif values == "few":  # many ties
        w = rng.integers(0, 3, (hkv, batch.total)).astype(np.float64)
    else:  # everything that a float can be
        w = rng.choice([0.0, -0.0, 1.0, -1.0, np.inf, -np.inf, np.nan, 1e-45, 3e38, -2.5], (hkv, batch.total))
    pos = np.zeros((hkv, batch.total), np.int64)
    for b, n in enumerate(lens):
        s = int(batch.kv_indptr_host[b])
        for g in range(hkv):  # distinct, in any order of rows
            pos[g, s:s + n] = rng.permutation(2 * n)[:n]
    return batch, K, V, w.astype(np.float32), pos.astype(np.int32)


@pytest.mark.parametrize("values", ["pareto", "few", "odd"])
@pytest.mark.parametrize("lens,keep,room,recent,spare", [
    ([1000, 1, 0, 5000], [250, 1, 4, 1024], [250, 3, 7, 2000], 64, 0),
    ([1025, 300], [1024, 299], [1024, 299], 0, 0),
    ([2000, 50], [10, 0], [10, 5], 100, 30),        # fewer kept than are recent; none kept
    ([64, 3000], [9999, 2999], [64, 5], 1, 0),      # more asked than there are, less room than asked
    ([20000], [5000], [5000], 500, 0),
])
def test_evict(values, lens, keep, room, recent, spare):
    import paper_2502_12216_amd as T
    hkv = 3
    batch, K, V, w, pos = _cache_inputs(lens, hkv, 11, spare, values)
    dest = T.RaggedBatch([0] * len(lens), hkv, hkv, capacities=room)
    ev = T.CacheEvictor(batch, dest, recent)
    Ko, Vo = (torch.full((hkv, dest.total, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    wo = torch.full((hkv, dest.total), -3.0, device=DEV)
    po = torch.full((hkv, dest.total), -9, dtype=torch.int32, device=DEV)
    newest = np.array([2 * max(n, 1) - 1 for n in lens], np.int32)
    for use_pos in (True, False):
        kw = dict(positions=torch.as_tensor(pos, device=DEV), newest=torch.as_tensor(newest, device=DEV)) if use_pos else {}
        ev(K, V, torch.as_tensor(w, device=DEV), torch.tensor(keep, dtype=torch.int32, device=DEV), Ko, Vo, wo, po, **kw)
        torch.cuda.synchronize()
        kept = [min(n, k, r) for n, k, r in zip(lens, keep, room)]
        assert dest.seq_len.tolist() == kept
        for b, n in enumerate(lens):
            s, o = int(batch.kv_indptr_host[b]), int(dest.kv_indptr_host[b])
            for g in range(hkv):
                p = pos[g, s:s + n] if use_pos else np.arange(n, dtype=np.int32)
                rows = np.sort(R.ranking(w[g, s:s + n], p, newest[b] if use_pos else n - 1, recent)[:kept[b]])
                to = slice(o, o + kept[b])
                assert po[g, to].cpu().numpy().tolist() == p[rows].tolist(), (b, g)
                at = torch.as_tensor(s + rows, device=DEV)
                assert torch.equal(Ko[g, to], K[g, at]) and torch.equal(Vo[g, to], V[g, at])
                assert np.array_equal(wo[g, to].cpu().numpy(), w[g, s + rows], equal_nan=True)
                behind = slice(o + kept[b], int(dest.kv_indptr_host[b + 1]))
                assert (Ko[g, behind] == 7).all() and (Vo[g, behind] == 7).all()
                assert (wo[g, behind] == -3).all() and (po[g, behind] == -9).all()


@pytest.mark.parametrize("values", ["pareto", "few", "odd"])
def test_insert(values):
    """Sequences with room, full ones, one where every row is recent, one without rows."""
    import paper_2502_12216_amd as T
    hkv, caps, lens, recent = 3, [300, 64, 1000, 20, 0, 7], [300, 60, 1000, 20, 0, 0], 30
    batch, K, V, w, pos = _cache_inputs(caps, hkv, 21, 0, values)
    for b in range(6):  # (the sequence of 20 rows: all recent)
        s, n = int(batch.kv_indptr_host[b]), caps[b]
        if n == 20:
            pos[:, s:s + n] = 20 + np.argsort(np.random.default_rng(1).random((hkv, n)), axis=1)
    batch = T.RaggedBatch(lens, hkv, hkv, capacities=caps)
    ins = T.TokenInserter(batch, recent)
    wt, pt = torch.as_tensor(w, device=DEV), torch.as_tensor(pos, device=DEV)
    for step in range(4):
        k, v = _randn(50 + step, 6, hkv, 128), _randn(60 + step, 6, hkv, 128)
        newest = np.array([2 * c + step for c in caps], np.int32)
        before = [x.clone() for x in (K, V, wt, pt)]
        n_now = batch.seq_len.tolist()
        rows = ins(k, v, K, V, wt, pt, torch.as_tensor(newest, device=DEV))
        torch.cuda.synchronize()
        for b in range(6):
            s, n = int(batch.kv_indptr_host[b]), n_now[b]
            for g in range(hkv):
                if caps[b] == 0:
                    assert int(rows[b, g]) == -1
                    continue
                if n < caps[b]:
                    want = n
                else:
                    want = int(R.ranking(before[2][g, s:s + n].cpu().numpy(), before[3][g, s:s + n].cpu().numpy(), newest[b], recent)[-1])
                assert int(rows[b, g]) == want, (step, b, g)
                for x in before[:2]:
                    x[g, s + want] = (k if x is before[0] else v)[b, g]
                before[2][g, s + want], before[3][g, s + want] = 0.0, int(newest[b])
        for x, y in zip(before, (K, V, wt, pt)):
            assert torch.equal(torch.nan_to_num(x.float(), 5.5), torch.nan_to_num(y.float(), 5.5))
        assert batch.seq_len.tolist() == [min(n + 1, c) for n, c in zip(n_now, caps)]


def _loop(cache, lens, hq, hkv, steps, check=True, decode=None):
    """Prompts into `cache`, then `steps` of append and decode; every stage against 64 bits, from the rows held."""
    q = [_randn(100 + b, n, hq, 128) for b, n in enumerate(lens)]
    K = [_randn(200 + b, hkv, n, 128) for b, n in enumerate(lens)]
    V = [_randn(300 + b, hkv, n, 128) for b, n in enumerate(lens)]
    out = cache.prefill(q, K, V)
    torch.cuda.synchronize()
    G, at, hist = hq // hkv, 0, [[K[b].clone(), V[b].clone()] for b in range(len(lens))]
    for b, n in enumerate(lens):
        pos = torch.arange(n, device=DEV)
        for h in range(hq):
            o, _, p, ma, off = R.attend(q[b][:, h], K[b][h // G], V[b][h // G], pos, pos, pos[None] <= pos[:, None],
                                        cache.mod.cap, float(cache.mod.slopes[h]))
            R.close(out[at:at + n, h], o, R.tolerance_bf16(ma, off, o), f"prefill b={b} h={h}")
        at += n
    outs = []
    for step in range(steps):
        k, v = _randn(400 + step, len(lens), hkv, 128), _randn(500 + step, len(lens), hkv, 128)
        cache.append(k, v)
        for b in range(len(lens)):
            hist[b] = [torch.cat([x, y[b][:, None]], 1) for x, y in zip(hist[b], (k, v))]
        qd = _randn(600 + step, len(lens), hq, 128)
        before = cache.weights.clone()
        o = (decode or cache.decode)(qd).clone()
        outs.append(o)
        torch.cuda.synchronize()
        for b in range(len(lens)):
            held = int(cache.batch.seq_len[b])
            assert held == min(cache.budget, lens[b] + step + 1) == cache.batch.seq_lens[b]
            s, new = int(cache.batch.kv_indptr_host[b]), lens[b] + step
            assert int(cache.newest[b]) == new
            for g in range(hkv):
                r = slice(s, s + held)
                pos = cache.positions[g, r].long()
                assert len(set(pos.tolist())) == held and int(pos.max()) == new
                recent = set(range(max(0, new - cache.recent + 1), new + 1))
                assert recent <= set(pos.tolist())
                # every row is the token that its position names
                assert torch.equal(cache.K[g, r], hist[b][0][g, pos]) and torch.equal(cache.V[g, r], hist[b][1][g, pos])
                added = torch.zeros(held, dtype=torch.float64, device=DEV)
                for h in range(g * G, (g + 1) * G):
                    ref, _, p, ma, off = R.attend(qd[b, h:h + 1], cache.K[g, r], cache.V[g, r],
                                                  torch.tensor([new], device=DEV), pos,
                                                  torch.ones(1, held, dtype=torch.bool, device=DEV), cache.mod.cap,
                                                  float(cache.mod.slopes[h]))
                    R.close(o[b, h:h + 1], ref, R.tolerance_fp32(ma, off, ref), f"decode step {step} b={b} h={h}")
                    added += p[0]
                want = before[g, r].double() + added
                R.close(cache.weights[g, r], want, 1e-5 * want.abs() + 1e-12, "sums")
    return outs


def test_evicting_cache_run():
    import paper_2502_12216_amd as T
    _loop(T.EvictingCache(8, 2, 3, 96, recent=16, window=20, cap=30.0, slopes=R.slopes(8)), [300, 90, 96], 8, 2, 12)


def test_evicting_cache_step_captured_and_replayed():
    """append and decode in a graph, replayed with eager work between, against an eager run on the same inputs."""
    import paper_2502_12216_amd as T
    def make():
        c = T.EvictingCache(8, 2, 2, 64, recent=8, slopes=R.slopes(8))
        lens = [200, 60]
        c.prefill([_randn(1 + b, n, 8, 128) for b, n in enumerate(lens)], [_randn(3 + b, 2, n, 128) for b, n in enumerate(lens)],
                  [_randn(5 + b, 2, n, 128) for b, n in enumerate(lens)])
        return c
    eager, graphed = make(), make()
    k, v, q = (torch.zeros(2, h, 128, dtype=torch.bfloat16, device=DEV) for h in (2, 2, 8))
    state = [graphed.K, graphed.V, graphed.weights, graphed.positions, graphed.newest, graphed.batch.seq_len]
    saved = [x.clone() for x in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (the first call sizes the workspace)
        graphed.append(k, v)
        graphed.decode(q)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.append(k, v)
        out = graphed.decode(q)
    for x, y in zip(state, saved):
        x.copy_(y)
    for step in range(10):
        kk, vv, qq = (_randn(70 + 3 * step + i, 2, h, 128) for i, h in enumerate((2, 2, 8)))
        eager.append(kk, vv)
        ref = eager.decode(qq).clone()
        for a, b in ((k, kk), (v, vv), (q, qq)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref), step
        for a, b in zip(state, (eager.K, eager.V, eager.weights, eager.positions, eager.newest, eager.batch.seq_len)):
            assert torch.equal(a, b), step


@pytest.mark.parametrize("values", ["pareto", "few", "odd"])
@pytest.mark.parametrize("lens,keep,room,recent,spare", [
    ([70000, 16385, 0, 5, 4096], [20000, 4000, 3, 3, 4096], [20000, 4000, 3, 5, 4096], 300, 0),  # several workgroups each
    ([131072, 65537], [131071, 1], [131071, 1], 0, 7),
    ([40000], [39999], [39999], 39000, 0),
    ([17000] + [100] * 10, [4000] + [99] * 10, [4000] + [99] * 10, 64, 0),      # many sequences: one workgroup each
    ([66000] + [90] * 10, [9000] + [50] * 10, [9000] + [50] * 10, 64, 3),
    ([66000] + [9] * 22, [9000] + [5] * 22, [9000] + [5] * 22, 64, 3),
])
def test_evict_long_sequences(values, lens, keep, room, recent, spare):
    test_evict(values, lens, keep, room, recent, spare)


@pytest.mark.parametrize("hkv", [1, 3, 5, 16, 20])
@pytest.mark.parametrize("caps,lens", [([40, 300, 0, 7], [40, 299, 0, 7]), ([9000, 5], [9000, 2]), ([5000, 4097], [5000, 4097])])
def test_insert_heads_and_lengths(hkv, caps, lens):
    """Heads that do not divide the waves, and caches on both sides of the one-launch limit: two tokens, ties included."""
    import paper_2502_12216_amd as T
    B = len(caps)
    _, K, V, w, pos = _cache_inputs(caps, hkv, 31, 0, "few")
    batch = T.RaggedBatch(lens, hkv, hkv, capacities=caps)
    ins = T.TokenInserter(batch, 3)
    wt, pt = torch.as_tensor(w, device=DEV), torch.as_tensor(pos, device=DEV)
    for step in range(2):
        k, v = _randn(70 + step, B, hkv, 128), _randn(80 + step, B, hkv, 128)
        newest = np.array([2 * c + step for c in caps], np.int32)
        now, w0, p0 = batch.seq_len.tolist(), wt.cpu().numpy().copy(), pt.cpu().numpy().copy()
        K0, V0 = K.clone(), V.clone()
        rows = ins(k, v, K, V, wt, pt, torch.as_tensor(newest, device=DEV)).tolist()
        torch.cuda.synchronize()
        for b in range(B):
            s, n = int(batch.kv_indptr_host[b]), now[b]
            for g in range(hkv):
                if caps[b] == 0:
                    assert rows[b][g] == -1
                    continue
                want = n if n < caps[b] else int(R.ranking(w0[g, s:s + n], p0[g, s:s + n], newest[b], 3)[-1])
                assert rows[b][g] == want, (step, b, g)
                K0[g, s + want], V0[g, s + want] = k[b, g], v[b, g]
                w0[g, s + want], p0[g, s + want] = 0.0, newest[b]
        assert torch.equal(K, K0) and torch.equal(V, V0)
        assert np.array_equal(wt.cpu().numpy(), w0) and np.array_equal(pt.cpu().numpy(), p0)
        assert batch.seq_len.tolist() == [min(n + 1, c) for n, c in zip(now, caps)]
