"""Every form of the prompt attention and of a shared prefix's (32, 64, 128 or 256 rows to an item, keys split among
workgroups or not) against the plain 64-bit implementation.  The host takes the form by an estimate of the time, which is worked out here
again: each case names its form, and the size of the workspace, which follows from it, has to agree."""
import math

import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attention import DEV, _documents, _randn, check_prompt
from tests.test_gpu_attention_tiles import test_shared_prefix_row_tiles as _shared_row_tiles

SPLITS = (1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 56, 64)
COSTS = ((1.3, 0.88, 128), (2.0, 1.9, 128), (2.5, 2.3, 128), (2.0, 1.85, 64))  # item, round (us), keys of a round
SHARED_COSTS = ((1.3, 1.05, 128), (2.0, 1.9, 128), (2.5, 1.7, 64), (2.0, 1.8, 32))


def form(lens, new, hq, hkv):
    """(rows to an item, splits of the keys) with the least estimated time."""
    most = max(lens)
    return _least(sum(new) * (hq // hkv), len(lens), hkv, max(1.0, most - 0.5 * min(max(new), most)), most, sum(lens), COSTS)


def shared_form(prefix, members, hq, hkv):
    return _least(members * (hq // hkv), 1, hkv, prefix, prefix, prefix, SHARED_COSTS)


def _least(rows, sources, hkv, mean, most, total, costs):
    memory = total * hkv * 512 / 6e6
    best = None
    for v, (item, step, keys) in enumerate(costs):
        items = max(sources, -(-rows // (32 << v))) * hkv
        for s in SPLITS:
            if s > 1 and s * keys > most:
                break
            run = max(math.ceil(most / (s * keys)) * step + item, math.ceil(items * s / 256) * (mean / (s * keys) * step + item))
            t = max(run, memory) + 0.5 * min(run, memory)
            if costs is SHARED_COSTS:
                t += 0.1 * s
            elif s > 1:
                t += 4 + 0.15 * s + rows * hkv * s * (2 * 520) / 4.5e6
            if best is None or t < best[0]:
                best = (t, 32 << v, s)
    return best[1:]


def tiles(lens, new, hq, hkv):
    return sum(new) * (hq // hkv) // form(lens, new, hq, hkv)[0] + len(lens)


def workspace(lens, new, hq, hkv):
    G, total, splits = hq // hkv, sum(lens), form(lens, new, hq, hkv)[1]

    def take(at, size):
        return -(-(at + size) // 256) * 256
    at = behind = take(0, -(-max(lens) // 64) * len(lens) * 8)
    for size in ([sum(new) * hq * splits * 512, sum(new) * hq * splits * 8] if splits > 1 else []):
        at = take(at, size)
    for size in (16, 4, 16):
        at = take(at, tiles(lens, new, hq, hkv) * size)
    items, rows = max(1, (total + 255) // 256) * hkv, max(new) * G  # the sums of the accumulated weights' splits
    weight_splits = max(1, min(max(min(4096 // items, rows // 512), min(512 // items, rows // 128)), 64))
    if weight_splits > 1:
        behind = take(behind, weight_splits * hkv * total * 4)
    return max(256, at, behind)


def ordered(lens, new, hq, hkv):
    """Whether the row tiles of documents are put in order first."""
    return form(lens, new, hq, hkv) == (256, 1) and tiles(lens, new, hq, hkv) * hkv > 384 and max(lens) > 256


# form, split or not, ordered or not
CASES = [
    ((32, False, False), [300, 200], [300, 200], 4, 2),
    ((32, False, False), [82, 80, 82, 1, 82, 77, 82, 82, 82], [82, 80, 82, 1, 82, 77, 82, 82, 82], 32, 16),
    ((32, True, False), [2100, 900], [64, 5], 8, 2),
    ((64, False, False), [700, 700, 701], [700, 700, 690], 12, 6),
    ((64, False, False), [400, 333, 397], [300, 290, 299], 32, 8),
    ((128, False, False), [400, 1, 0, 399, 400, 380], [200, 1, 0, 200, 200, 199], 32, 8),
    ((128, False, False), [2100, 2033, 2055], [1500, 1400, 1499], 6, 6),
    ((128, False, False), [1026, 1000] * 6, [115, 114] * 6, 64, 16),
    ((128, True, False), [3999], [301], 16, 2),
    ((128, True, False), [3558] * 12, [56] * 12, 32, 8),
    ((256, False, False), [400, 390, 400, 400, 370, 400], [200, 190, 200, 200, 170, 200], 32, 8),
    ((256, False, False), [120] * 20, [120] * 20, 32, 8),
    ((256, False, True), [1300, 0, 900, 1201], [1300, 0, 900, 1201], 32, 8),
    ((256, False, True), [2500, 2400, 2500] * 2, [2500, 2400, 2450] * 2, 8, 2),
    ((256, True, False), [6000], [3000], 4, 2),
    ((256, True, False), [20000], [520], 16, 2),
]
MASKS = [dict(), dict(cap=30.0, page=16), dict(alibi=True, prefix=100, spare=3), dict(docs=60), dict(page=64, alibi=True),
         dict(docs=300, page=7, alibi=True, cap=3.0), dict(docs=2000, prefix=700)]


def _known(case):
    named, *shape = case
    r, s = form(*shape)
    assert (r, s > 1, ordered(*shape)) == named
    return shape


@pytest.mark.parametrize("case", CASES)
def test_cases_take_the_forms_that_they_name(case):
    """(On the CPU: the workspace's size is worked out on the host.)"""
    import paper_2502_12216_amd as T
    lens, new, hq, hkv = _known(case)
    att = T.PromptAttention(T.RaggedBatch(lens, hq, hkv, device="cpu"), new)
    assert att.workspace.numel() == workspace(lens, new, hq, hkv)


def test_cases_cover_every_form():
    assert {case[0][:2] for case in CASES} == {(r, s) for r in (32, 64, 128, 256) for s in (False, True)} - {(64, True)}


@pytest.mark.gpu
@pytest.mark.parametrize("kw", MASKS)
@pytest.mark.parametrize("case", CASES)
def test_prompt_forms(case, kw):
    lens, new, hq, hkv = _known(case)
    if "prefix" in kw:
        kw = dict(kw, prefix=[kw["prefix"] + 37 * b for b in range(len(lens))])
    check_prompt(lens, new, hq, hkv, **kw)


def check_spoilt(lens, new, hq, hkv, spoil, page, docs=0, alibi=False):
    """Values that are not finite, against the formula.  An infinity gives itself where its weight is in the range of
    32 bits (here: above 2^-100), below it itself or NaN (0 times it); every other value is as without it."""
    import paper_2502_12216_amd as T
    batch = T.RaggedBatch(lens, hq, hkv)
    K, V, q = _randn(1, hkv, batch.total, 128), _randn(2, hkv, batch.total, 128), _randn(3, sum(new), hq, 128, scale=2.0)
    spoil(K, V)
    document = torch.cat([torch.as_tensor(_documents(n, docs, 1), device=DEV) for n in lens]) if docs else None
    sl = R.slopes(hq) if alibi else None
    att, mod = T.PromptAttention(batch, new), T.ScoreMod(slopes=sl, documents=document)
    if page:
        kp, table = R.pages(K, lens, page, 1)
        out, lse = att.paged(q, T.PagedCache(kp, R.pages(V, lens, page, 1)[0], table), mod)
    else:
        out, lse = att(q, K, V, mod)
    torch.cuda.synchronize()
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        r = slice(int(batch.kv_indptr_host[b]), int(batch.kv_indptr_host[b + 1]))
        kpos, qpos = torch.arange(n, device=DEV), torch.arange(n - m, n, device=DEV)
        seen = kpos[None] <= qpos[:, None]
        if docs:
            seen = seen & (document[r][qpos][:, None] == document[r][None])
        for h in range(hq):
            g = h * hkv // hq
            v = V[g, r].double()
            o, l, p, ma, off = R.attend(q[at:at + m, h], K[g, r], torch.nan_to_num(v, 0.0, 0.0, 0.0), qpos, kpos, seen, 0.0,
                                        float(sl[h]) if alibi else 0.0)
            R.close(lse[h, at:at + m], l, R.tolerance_lse(off, l), f"lse b={b} h={h}")

            def some(keys, value):  # whether one of a query's `keys` has the value, per dimension
                return keys.double() @ value.double() > 0
            got, inf = out[at:at + m, h].double(), float("inf")
            up, down = some(seen, v == inf), some(seen, v == -inf)
            nan = torch.isnan(l)[:, None] | some(seen, torch.isnan(v))
            finite = ~(nan | up | down)
            assert torch.isnan(got[nan]).all(), (b, h)
            for value, here, other in ((inf, up, down), (-inf, down, up)):
                sure, may = some(p > 2.0 ** -100, v == value) & ~nan & ~other, here & ~nan & ~other
                assert (got[sure] == value).all(), (b, h)
                assert (torch.isnan(got[may]) | (got[may] == value)).all(), (b, h)
            assert not torch.isfinite(got[up & down]).any(), (b, h)
            R.close(torch.where(finite, got, 0.0), torch.where(finite, o, 0.0),
                    torch.where(finite, R.tolerance_bf16(ma, off, o), 1e-30), f"out b={b} h={h}")
        at += m


@pytest.mark.gpu
@pytest.mark.parametrize("page", [0, 24])
@pytest.mark.parametrize("kw", [dict(docs=25), dict(), dict(alibi=True)])
@pytest.mark.parametrize("case", [c for c in CASES if max(c[1]) < 5000])
def test_prompt_forms_with_values_that_are_not_finite(case, kw, page):
    """In places that some queries see, that others do not, and that nobody sees: the items are computed again."""
    lens, new, hq, hkv = _known(case)

    def spoil(K, V):
        n = lens[0]
        for i, value in enumerate((float("nan"), float("inf"), -float("inf"))):
            V[i::3, n // 2 + 11 + i, 5 * i:5 * i + 2] = value
            V[0, max(n - 60, 0) + 3 * i] = value
            K[1, max(n - 100, 30) + 7 * i, 3] = value
    check_spoilt(lens, new, hq, hkv, spoil, page, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(docs=200), dict(alibi=True)])
def test_split_256_row_form_with_values_that_are_not_finite(kw):
    """The last queries of a long sequence in pages, of which some see what is spoilt."""
    lens, new, hq, hkv = _known(next(c for c in CASES if c[0] == (256, True, False) and c[2] == [520]))

    def spoil(K, V):
        V[0, 19990, 7] = float("nan")
        V[1, 19000:19900:50, 9] = float("inf")
        V[1, 5, 30] = -float("inf")
        K[1, 19970, 3] = float("nan")
    check_spoilt(lens, new, hq, hkv, spoil, 64, **kw)


SHARED = [  # form, tokens of the prefix, its sequences, heads
    ((32, False), 5, 300, 8, 8), ((32, True), 333, 3, 8, 2), ((64, False), 100, 512, 32, 8), ((64, True), 1000, 150, 32, 8),
    ((128, False), 45, 262, 64, 8), ((128, True), 1000, 200, 32, 8), ((256, False), 17, 262, 64, 8), ((256, True), 100, 512, 64, 8),
]


def _known_shared(case):
    (rows, split), *shape = case
    r, s = shared_form(*shape)
    assert (r, s > 1) == (rows, split)
    return shape


@pytest.mark.parametrize("case", SHARED)
def test_shared_cases_take_the_forms_that_they_name(case):
    """(On the CPU.)  The workspace is that of a decode and the sums of every split."""
    import ctypes

    import paper_2502_12216_amd as T
    prefix, members, hq, hkv = _known_shared(case)
    batch = T.RaggedBatch([i % 4 for i in range(members)], hq, hkv, device="cpu")
    shape = batch.struct()
    rest = T.SharedPrefixDecoder(batch, [prefix], [0] * members).workspace.numel() - \
        T.lib().tactic_scored_decode_workspace_size(ctypes.byref(shape), 0)
    assert 0 <= rest - shared_form(prefix, members, hq, hkv)[1] * members * hq * (512 + 8) < 512


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(), dict(cap=20.0), dict(page=16, alibi=True)])
@pytest.mark.parametrize("case", [c for c in SHARED if c[0] in ((32, False), (32, True), (128, False), (256, False))])
def test_shared_forms(case, kw):
    _shared_row_tiles(*_known_shared(case), kw)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [0, 24])
@pytest.mark.parametrize("scale", [1.0, 64.0])
@pytest.mark.parametrize("case", SHARED)
def test_shared_forms_with_values_that_are_not_finite(case, scale, page):
    """Every sequence sees all of the prefix: what is not finite there reaches each of them, in full tiles and in the
    last one, which is looked over; with scores of hundreds (scale) most weights are below the range of 32 bits."""
    import paper_2502_12216_amd as T
    n, members, hq, hkv = _known_shared(case)
    lens = [i % 3 for i in range(members)]
    batch = T.RaggedBatch(lens, hq, hkv)
    Kp, Vp, q = _randn(1, hkv, n, 128, scale=scale), _randn(2, hkv, n, 128), _randn(3, members, hq, 128, scale=2.0)
    K, V = _randn(4, hkv, batch.total, 128, scale=scale), _randn(5, hkv, batch.total, 128)
    Vp[0, n - 1, 3] = float("inf")
    Vp[0, n // 2, 7] = float("nan")
    Vp[1, 0, 9] = -float("inf")
    Vp[1, n - 2, 11], Vp[1, n // 3, 11] = float("inf"), -float("inf")
    dec = T.SharedPrefixDecoder(batch, [n], [0] * members)
    if page:
        parts = []
        for k, v, m in ((Kp, Vp, [n]), (K, V, lens)):
            a, table = R.pages(k, m, page, 1)
            parts.append(T.PagedCache(a, R.pages(v, m, page, 1)[0], table))
        out, lse = dec.paged(q, *parts)
    else:
        out, lse = dec(q, Kp, Vp, K, V)
    torch.cuda.synchronize()
    own = torch.as_tensor(lens, device=DEV)
    of = torch.repeat_interleave(torch.arange(members, device=DEV), own)
    seen = torch.cat([torch.ones(members, n, dtype=torch.bool, device=DEV), of[None] == torch.arange(members, device=DEV)[:, None]], 1)
    pos = torch.zeros(max(members, n + len(of)), dtype=torch.int64, device=DEV)
    for h in range(hq):
        g = h * hkv // hq
        v = torch.cat([Vp[g], V[g]]).double()
        o, l, p, ma, off = R.attend(q[:, h], torch.cat([Kp[g], K[g]]), torch.nan_to_num(v, 0.0, 0.0, 0.0), pos[:members],
                                    pos[:n + len(of)], seen)
        R.close(lse[:, h], l, R.tolerance_lse(off, l), f"lse h={h}")
        got, nan = out[:, h].double(), torch.isnan(v).any(0)
        up, down = (v == float("inf")).any(0), (v == -float("inf")).any(0)
        assert torch.isnan(got[:, nan | (up & down)]).all()
        finite = ~(nan | up | down)
        R.close(got[:, finite], o[:, finite], R.tolerance_fp32(ma, off, o)[:, finite], f"out h={h}")
        for value, only in ((float("inf"), up & ~down), (-float("inf"), down & ~up)):
            x, weight = got[:, only], (p @ (v == value).double())[:, only]
            assert ((x == value) | (torch.isnan(x) & (weight < 2.0 ** -100))).all(), h


@pytest.mark.gpu
def test_lengths_that_are_nothing():
    """No queries at all, or queries without any tokens: nothing written, and zeros."""
    import paper_2502_12216_amd as T
    batch = T.RaggedBatch([0, 0], 8, 2)
    rows = torch.zeros(2, 0, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = T.PromptAttention(batch, [0, 0])(torch.zeros(0, 8, 128, dtype=torch.bfloat16, device="cuda"), rows, rows)
    assert out.shape == (0, 8, 128) and lse.shape == (8, 0)
    out, lse = T.PromptAttention(batch, [3, 0])(torch.ones(3, 8, 128, dtype=torch.bfloat16, device="cuda"), rows, rows)
    torch.cuda.synchronize()
    assert not out.any() and (lse == -float("inf")).all()
