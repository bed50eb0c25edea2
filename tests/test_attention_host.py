"""Host-side checks of the calls beside the sparse decode: every refusal comes
before any launch, so no GPU is needed (fake device pointers are never read)."""
import ctypes

import pytest
import torch

import paper_2502_12216_amd as T
from paper_2502_12216_amd import _capi as C

FAKE, OTHER = 0x1000, 0x2000
NAN = float("nan")


def _shape(B=2, Hq=8, Hkv=2, d=128, total=1000, nmax=700, indptr=FAKE, lens=None):
    return C.KVShape(B, Hq, Hkv, d, total, nmax, indptr, lens)


def _queries(total=100, most=60, indptr=FAKE):
    return C.QueryShape(total, most, indptr)


def _prefixes(n=2, members=2, total=500, longest=300, indptr=FAKE, of=FAKE, ids=FAKE, mptr=FAKE, all_members=2):
    return C.Prefixes(n, members, total, longest, indptr, of, ids, mptr, all_members)


def _paged(K=FAKE, page=16, pages=64, num=200):
    return C.PagedKV(K, FAKE, FAKE, None, page, pages, num)


R = ctypes.byref
BIG = 1 << 40


def prompt(shape=None, queries=None, mod=None, q=FAKE, K=FAKE, V=FAKE, out=FAKE, lse=None, ws=FAKE, n=BIG):
    shape, queries, mod = shape or _shape(), queries or _queries(), mod or C.ScoreMod()
    return C.lib().tactic_prompt_attention(q, K, V, R(shape), R(queries), R(mod), out, lse, ws, n, None)


def weights(shape=None, queries=None, mod=None, q=FAKE, K=FAKE, lse=FAKE, window=0, w=FAKE, ws=FAKE, n=BIG):
    shape, queries, mod = shape or _shape(), queries or _queries(), mod or C.ScoreMod()
    return C.lib().tactic_prompt_weights(q, K, R(shape), R(queries), R(mod), lse, window, w, ws, n, None)


def scored(shape=None, mod=None, rows=None, q=FAKE, K=FAKE, out=FAKE, w=None, ws=FAKE, n=BIG):
    shape, mod, rows = shape or _shape(), mod or C.ScoreMod(), rows or C.TokenRows()
    return C.lib().tactic_scored_decode(q, K, FAKE, R(shape), R(mod), R(rows), out, None, w, ws, n, None)


def shared(shape=None, pre=None, mod=None, q=FAKE, Kp=FAKE, K=FAKE, out=FAKE, ws=FAKE, n=BIG):
    shape, pre, mod = shape or _shape(), pre or _prefixes(), mod or C.ScoreMod()
    return C.lib().tactic_shared_decode(q, Kp, FAKE, K, FAKE, R(shape), R(pre), R(mod), out, None, ws, n, None)


def evict(shape=None, K=FAKE, w=FAKE, keep=FAKE, recent=5, indptr=FAKE, total=100, most=60, Ko=OTHER, wo=OTHER, lens=FAKE,
          ws=FAKE, n=BIG):
    return C.lib().tactic_evict(K, FAKE, R(shape or _shape()), w, FAKE, keep, None, recent, indptr, total, most, Ko, OTHER,
                                wo, OTHER, lens, ws, n, None)


def insert(shape=None, k=FAKE, newest=FAKE, recent=5, lens=FAKE, K=FAKE, rows=FAKE):
    return C.lib().tactic_insert_token(k, FAKE, newest, recent, R(shape or _shape(lens=FAKE)), lens, K, FAKE, FAKE, FAKE,
                                       rows, None)


BAD_SHAPES = [(dict(B=0), 1), (dict(Hq=6, Hkv=4), 1), (dict(Hq=6, Hkv=2), 2), (dict(d=64), 2), (dict(indptr=None), 1),
              (dict(total=10, nmax=20), 1), (dict(total=1 << 40, nmax=1 << 31), 2), (dict(B=4097, Hq=1, Hkv=1), 2)]


@pytest.mark.parametrize("call", [prompt, weights, scored, shared, evict, insert])
@pytest.mark.parametrize("kw,code", BAD_SHAPES)
def test_bad_shapes(call, kw, code):
    assert call(shape=_shape(**kw)) == code, C.lib().tactic_last_error()


@pytest.mark.parametrize("call", [prompt, weights, scored, shared])
@pytest.mark.parametrize("cap", [-1.0, NAN, float("inf")])
def test_bad_caps(call, cap):
    assert call(mod=C.ScoreMod(cap)) == 1
    assert b"cap" in C.lib().tactic_last_error()


@pytest.mark.parametrize("call", [prompt, weights])
@pytest.mark.parametrize("q,code", [(dict(indptr=None), 1), (dict(total=-1), 1), (dict(most=101), 1), (dict(total=121), 1),
                                    (dict(total=1 << 30, most=1 << 30), 2)])
def test_bad_queries(call, q, code):
    assert call(queries=_queries(**q)) == code


@pytest.mark.parametrize("call,kw,code", [
    (prompt, dict(q=None), 1), (prompt, dict(K=None), 1), (prompt, dict(V=None), 1), (prompt, dict(out=None), 1),
    (prompt, dict(ws=None), 3), (prompt, dict(n=100), 3),
    (weights, dict(q=None), 1), (weights, dict(K=None), 1), (weights, dict(lse=None), 1), (weights, dict(w=None), 1),
    (weights, dict(window=-1), 1), (weights, dict(n=10), 3),
    (scored, dict(q=None), 1), (scored, dict(K=None), 1), (scored, dict(out=None), 1), (scored, dict(ws=None), 3),
    (scored, dict(n=1000), 3), (scored, dict(mod=C.ScoreMod(0, None, FAKE)), 1),
    (scored, dict(rows=C.TokenRows(None, None, FAKE)), 1), (scored, dict(mod=C.ScoreMod(0, None, None, FAKE)), 1),
    (scored, dict(mod=C.ScoreMod(0, FAKE), rows=C.TokenRows(FAKE)), 1),
    (shared, dict(q=None), 1), (shared, dict(Kp=None), 1), (shared, dict(K=None), 1), (shared, dict(out=None), 1),
    (shared, dict(mod=C.ScoreMod(0, None, FAKE)), 2), (shared, dict(mod=C.ScoreMod(0, None, None, FAKE)), 2),
    (shared, dict(n=1000), 3), (shared, dict(pre=_prefixes(n=0)), 1), (shared, dict(pre=_prefixes(all_members=3)), 1),
    (shared, dict(pre=_prefixes(all_members=1)), 1), (shared, dict(pre=_prefixes(longest=501)), 1),
    (shared, dict(pre=_prefixes(indptr=None)), 1), (shared, dict(pre=_prefixes(of=None)), 1),
    (shared, dict(pre=_prefixes(ids=None)), 1), (shared, dict(pre=_prefixes(mptr=None)), 1),
    (shared, dict(pre=_prefixes(total=1 << 31, longest=(1 << 31) - 100)), 2),
    (evict, dict(K=None), 1), (evict, dict(w=None), 1), (evict, dict(keep=None), 1), (evict, dict(indptr=None), 1),
    (evict, dict(Ko=None), 1), (evict, dict(Ko=FAKE), 1), (evict, dict(wo=FAKE), 1), (evict, dict(lens=None), 1),
    (evict, dict(recent=-1), 1), (evict, dict(recent=(1 << 22) + 1), 1), (evict, dict(most=101), 1), (evict, dict(total=-1), 1),
    (evict, dict(n=10), 3), (evict, dict(total=1 << 32, most=1 << 31), 2),
    (insert, dict(k=None), 1), (insert, dict(newest=None), 1), (insert, dict(lens=OTHER), 1), (insert, dict(K=None), 1),
    (insert, dict(rows=None), 1), (insert, dict(recent=-1), 1),
])
def test_refusals(call, kw, code):
    assert call(**kw) == code, C.lib().tactic_last_error()


@pytest.mark.parametrize("kw,code", [(dict(K=None), 1), (dict(page=0), 1), (dict(pages=2), 1), (dict(num=0), 1),
                                     (dict(pages=1 << 28), 2), (dict(num=1 << 30), 2)])
def test_bad_pages(kw, code):
    L, bad, good, shape = C.lib(), _paged(**kw), _paged(), _shape()
    queries, mod, rows, pre = _queries(), C.ScoreMod(), C.TokenRows(), _prefixes()
    assert L.tactic_prompt_attention_paged(FAKE, R(bad), R(shape), R(queries), R(mod), FAKE, None, FAKE, BIG, None) == code
    assert L.tactic_scored_decode_paged(FAKE, R(bad), R(shape), R(mod), R(rows), FAKE, None, None, FAKE, BIG, None) == code
    for a, b in ((bad, good), (good, bad)):
        assert L.tactic_shared_decode_paged(FAKE, R(a), R(b), R(shape), R(pre), R(mod), FAKE, None, FAKE, BIG, None) == code


def test_workspace_sizes():
    L = C.lib()
    assert L.tactic_prompt_attention_workspace_size(R(_shape(d=64)), R(_queries())) == 0
    assert L.tactic_prompt_attention_workspace_size(R(_shape()), R(_queries(most=101))) == 0
    assert L.tactic_scored_decode_workspace_size(R(_shape(B=0)), 0) == 0
    assert L.tactic_shared_decode_workspace_size(R(_shape()), R(_prefixes(n=0))) == 0
    assert L.tactic_evict_workspace_size(R(_shape()), -1) == 0
    plain, summed = (L.tactic_scored_decode_workspace_size(R(_shape()), w) for w in (0, 1))
    assert summed - plain >= 1000 * 8 * 4  # a score per row and query head


def test_nothing_to_do_is_no_launch():
    empty = _queries(total=0, most=0)
    assert prompt(queries=empty, q=None, out=None, ws=None, n=0) == 0
    assert weights(queries=empty, q=None, lse=None, ws=None, n=0) == 0
    assert weights(shape=_shape(total=0, nmax=0), K=None, w=None, ws=None, n=0) == 0


def test_python_refusals():
    cpu = dict(device="cpu")
    batch = T.RaggedBatch([5, 3], 8, 2, **cpu)
    with pytest.raises(ValueError, match="cap"):
        T.ScoreMod(cap=-1.0)
    with pytest.raises(ValueError, match="q_lens"):
        T.PromptAttention(batch, [5])
    with pytest.raises(ValueError, match="q_lens"):
        T.PromptAttention(batch, [5, -1])
    for kw in (dict(prefix_of=[0]), dict(prefix_of=[0, 2]), dict(prefix_lens=[]), dict(prefix_lens=[3, -1])):
        with pytest.raises(ValueError, match="prefix"):
            T.SharedPrefixDecoder(batch, **{**dict(prefix_lens=[7, 9], prefix_of=[0, 1]), **kw})
    with pytest.raises(ValueError, match="capacities"):
        T.CacheEvictor(batch, T.RaggedBatch([1, 1], 8, 2, **cpu), 0)
    with pytest.raises(ValueError, match="same"):
        T.CacheEvictor(batch, T.RaggedBatch([1], 8, 2, capacities=[4], **cpu), 0)
    with pytest.raises(ValueError, match="capacities"):
        T.TokenInserter(batch, 0)
    with pytest.raises(ValueError, match="recent"):
        T.EvictingCache(8, 2, 1, 64, recent=64, **cpu)
    dec = T.ScoredDecoder(batch)
    q, kv = torch.zeros(2, 8, 128, dtype=torch.bfloat16), torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        dec(q, kv, kv)
    with pytest.raises(TypeError, match="bfloat16"):
        dec(q.float(), kv.float(), kv)


def test_evicting_cache_refuses_before_it_changes():
    """Prompts whose q, K and V differ in length, and tokens of another shape or type, leave the cache as it was."""
    import paper_2502_12216_amd as T
    c = T.EvictingCache(8, 2, 2, 16, recent=4, device="cpu")

    def kv(n):
        return torch.zeros(2, n, 128, dtype=torch.bfloat16)

    def q(n):
        return torch.zeros(n, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="every sequence"):
        c.prefill([q(3)], [kv(3), kv(5)], [kv(3), kv(5)])
    with pytest.raises(ValueError, match="one length"):
        c.prefill([q(5), q(3)], [kv(3), kv(5)], [kv(3), kv(5)])
    with pytest.raises(ValueError, match="one length"):
        c.prefill([q(3), q(5)], [kv(3), kv(5)], [kv(5), kv(3)])
    k = torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    for bad in (k[:1], k.float(), k.transpose(0, 1), torch.zeros(2, 3, 128, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            c.append(bad, bad)
        with pytest.raises(ValueError):
            c.append(k, bad)
    assert c.newest.tolist() == [-1, -1] and c.batch.seq_lens == [0, 0]


def test_evict_refuses_lengths_it_reads_while_it_writes_them():
    import paper_2502_12216_amd as T
    assert evict(shape=_shape(lens=FAKE), lens=FAKE) == 1
    assert b"seq_len" in C.lib().tactic_last_error()
    batch = T.RaggedBatch([3, 5], 2, 2, device="cpu", capacities=[8, 8])
    with pytest.raises(ValueError, match="another batch"):
        T.CacheEvictor(batch, batch, 0)


@pytest.mark.parametrize("call,names", [(prompt, ("q", "K", "V", "out")), (weights, ("q", "K")), (scored, ("q", "K", "out")),
                                        (shared, ("q", "Kp", "K", "out")), (evict, ("K", "Ko")), (insert, ("k", "K"))])
def test_rows_off_their_alignment(call, names):
    """Rows are read 16 bytes at a time."""
    for name in names:
        for off in (2, 8):
            assert call(**{name: FAKE + off}) == 1, name
            assert b"16-byte" in C.lib().tactic_last_error()
