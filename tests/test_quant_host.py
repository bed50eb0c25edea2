"""Host-side checks of the quantised cache's calls: every refusal comes before any launch, so no GPU is needed
(fake device pointers are never read)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2502_12216_amd as T
import quant_ref
from paper_2502_12216_amd import _capi as C

FAKE = 0x1000
R = ctypes.byref
BIG = 1 << 40
NAN = float("nan")


def _shape(B=2, Hq=8, Hkv=2, d=128, total=1000, nmax=700, indptr=FAKE, lens=None):
    return C.KVShape(B, Hq, Hkv, d, total, nmax, indptr, lens)


def _rows(total=100, most=60, indptr=FAKE):
    return C.QueryShape(total, most, indptr)


def _kv(K=FAKE, Ks=FAKE, V=FAKE, Vs=FAKE, bounds=FAKE, table=None, bits=8, block=64, page=16, pages=64, num=200):
    return C.QuantKV(K, Ks, V, Vs, bounds, table, bits, block, page, pages, num)


def write(shape=None, rows=None, kv=None, k=FAKE, v=FAKE):
    return C.lib().tactic_quant_write(k, v, R(shape or _shape()), R(rows or _rows()), R(kv or _kv()), None)


def read(shape=None, rows=None, kv=None, K=FAKE, V=FAKE):
    return C.lib().tactic_quant_read(R(kv or _kv()), R(shape or _shape()), R(rows or _rows()), K, V, None)


def select(shape=None, kv=None, q=FAKE, budget=8, first=1, last=2, blocks=FAKE, counts=FAKE, ws=FAKE, n=BIG):
    return C.lib().tactic_block_select(q, R(kv or _kv()), R(shape or _shape()), R(C.BlockParams(budget, first, last)), blocks,
                                       counts, ws, n, None)


def decode(shape=None, kv=None, mod=None, q=FAKE, blocks=None, counts=None, budget=0, out=FAKE, lse=None, ws=FAKE, n=BIG):
    return C.lib().tactic_quant_decode(q, R(kv or _kv()), R(shape or _shape()), R(mod or C.ScoreMod()), blocks, counts, budget, out,
                                       lse, ws, n, None)


BAD_SHAPES = [(dict(B=0), 1), (dict(Hq=6, Hkv=4), 1), (dict(Hq=24, Hkv=2), 2), (dict(d=64), 2), (dict(indptr=None), 1),
              (dict(total=10, nmax=20), 1), (dict(B=3000), 2)]


@pytest.mark.parametrize("call", [write, read, select, decode])
@pytest.mark.parametrize("kw,code", BAD_SHAPES)
def test_bad_shapes(call, kw, code):
    assert call(shape=_shape(**kw)) == code


@pytest.mark.parametrize("call", [write, read, decode])
@pytest.mark.parametrize("kw,code", [
    (dict(bits=5), 1), (dict(bits=0), 1), (dict(bits=16), 1), (dict(block=8), 1), (dict(block=48), 1), (dict(block=256), 1),
    (dict(block=-16), 1), (dict(block=0), 1), (dict(K=None), 1), (dict(Ks=None), 1), (dict(V=None), 1), (dict(Vs=None), 1),
    (dict(K=FAKE + 8), 1), (dict(V=FAKE + 4), 1), (dict(Ks=FAKE + 2), 1), (dict(Vs=FAKE + 1), 1), (dict(bounds=FAKE + 8), 1),
    (dict(table=FAKE, page=0), 1), (dict(table=FAKE, pages=0), 1), (dict(table=FAKE, num=0), 1),
    (dict(table=FAKE, page=16, pages=43), 1), (dict(table=FAKE, page=1 << 16, pages=1 << 15), 2),
    (dict(table=FAKE, num=1 << 27), 2),
])
def test_bad_caches(call, kw, code):
    assert call(kv=_kv(**kw)) == code


@pytest.mark.parametrize("call", [write, read])
@pytest.mark.parametrize("kw,code", [(dict(indptr=None), 1), (dict(total=-1), 1), (dict(most=-1), 1), (dict(most=101), 1),
                                     (dict(total=121), 1), (dict(total=1 << 31, most=1 << 30), 2)])
def test_bad_rows(call, kw, code):
    assert call(rows=_rows(**kw)) == code


@pytest.mark.parametrize("status", [
    lambda: write(k=None), lambda: write(v=None), lambda: write(k=FAKE + 8), lambda: write(v=FAKE + 2),
    lambda: read(K=None), lambda: read(V=None), lambda: read(K=FAKE + 8),
    lambda: select(q=None), lambda: select(blocks=None), lambda: select(counts=None), lambda: select(q=FAKE + 8),
    lambda: select(blocks=FAKE + 2), lambda: select(kv=_kv(bounds=None)), lambda: select(kv=_kv(bounds=None, block=0)),
    lambda: select(budget=0, first=0, last=0), lambda: select(first=-1), lambda: select(last=-1), lambda: select(budget=2),
    lambda: select(first=2 ** 31 - 1, last=2 ** 31 - 1),
    lambda: decode(q=None), lambda: decode(out=None), lambda: decode(q=FAKE + 8), lambda: decode(lse=FAKE + 2),
    lambda: decode(blocks=FAKE, budget=4), lambda: decode(counts=FAKE, budget=4),
    lambda: decode(blocks=FAKE, counts=FAKE, budget=0), lambda: decode(blocks=FAKE, counts=FAKE, budget=4, kv=_kv(bounds=None, block=0)),
    lambda: decode(mod=C.ScoreMod(NAN)), lambda: decode(mod=C.ScoreMod(-1.0)), lambda: decode(mod=C.ScoreMod(2.0 ** 121)),
])
def test_bad_arguments(status):
    assert status() == 1


def test_unsupported_scores_and_small_workspaces():
    assert decode(mod=C.ScoreMod(0.0, None, FAKE, None)) == 2 and decode(mod=C.ScoreMod(0.0, None, None, FAKE)) == 2
    need = C.lib().tactic_block_select_workspace_size(R(_shape()), 64)
    assert need > 0 and select(n=need - 1) == 3 and select(ws=None) == 3
    assert C.lib().tactic_block_select_workspace_size(R(_shape()), 8) == 0
    need = C.lib().tactic_dense_decode_workspace_size(R(_shape()))
    assert decode(n=need - 1) == 3 and decode(ws=None) == 3


def test_counts_past_the_limits():
    assert select(budget=(1 << 27) + 1) == 2 and select(budget=(1 << 31) - 1) == 2
    for total in (1 << 62, (1 << 63) - 1):
        assert write(rows=_rows(total=total, most=total)) == 2 and read(rows=_rows(total=total, most=total)) == 2


def test_arrays_that_overlap():
    """k, v and the cache's arrays (of 2000 rows of 128 bytes), each a byte too near to the next."""
    at = {"k": 1 << 24, "v": 2 << 24, "K": 3 << 24, "Ks": 4 << 24, "V": 5 << 24, "Vs": 6 << 24, "bounds": 7 << 24}
    size = {"k": 100 * 512, "v": 100 * 512, "K": 2000 * 128, "V": 2000 * 128, "Ks": 8000, "Vs": 8000, "bounds": (1000 // 64 + 2) * 1024}
    lib = C.lib()

    def refused(call, **over):  # (only calls that are: the pointers mean nothing)
        p = {**at, **over}
        kv = _kv(K=p["K"], Ks=p["Ks"], V=p["V"], Vs=p["Vs"], bounds=p["bounds"])
        status = (lib.tactic_quant_write(p["k"], p["v"], R(_shape()), R(_rows()), R(kv), None) if call == "write" else
                  lib.tactic_quant_read(R(kv), R(_shape()), R(_rows()), p["k"], p["v"], None))
        return status == 1 and "overlap" in lib.tactic_last_error().decode()

    for x in at:
        for y in at:
            if x != y:
                near, rows = at[y] + size[y] - 16, {x, y} & {"k", "v"}
                assert rows == {"k", "v"} or refused("write", **{x: near}), (x, y)  # (k and v of a write are both read)
                assert not rows or refused("read", **{x: near}), (x, y)


def test_nothing_to_do():
    assert write(rows=_rows(0, 0), k=None, v=None) == 0 and read(rows=_rows(0, 0), K=None, V=None) == 0
    assert write(shape=_shape(total=0, nmax=0), kv=_kv(K=None, Ks=None, V=None, Vs=None)) == 0


def test_objects_refuse():
    batch = T.RaggedBatch([5, 3], 8, 2, device="cpu", capacities=[10, 10])
    codes, scale = torch.zeros(2, 20, 128, dtype=torch.uint8), torch.zeros(2, 20, 4, dtype=torch.uint8)
    bounds = torch.zeros(2, 2, 2, 128, dtype=torch.bfloat16)
    for bad in (lambda: T.QuantizedCache(codes[..., :96], scale, codes, scale), lambda: T.QuantizedCache(codes[0], scale, codes, scale),
                lambda: T.QuantizedCache(codes, scale, codes, scale, bounds=bounds),
                lambda: T.QuantizedCache(codes, scale, codes, scale, block=16),
                lambda: T.QuantizedCache(codes, scale, codes, scale, bounds=bounds, block=24),
                lambda: T.QuantizedCache.empty(batch, 6), lambda: T.QuantizedCache.empty(batch, 8, 7),
                lambda: T.CacheQuantizer(batch, [1]), lambda: T.CacheQuantizer(batch, [1, -1]),
                lambda: T.BlockSelector(batch, 24, 4), lambda: T.BlockSelector(batch, 16, 2), lambda: T.BlockSelector(batch, 16, 0, 0, 0)):
        with pytest.raises(ValueError):
            bad()
    cache = T.QuantizedCache.empty(batch, 8, 16)
    assert cache.K.shape == (2, 20, 128) and cache.bounds.shape == (2, 3, 2, 128)
    with pytest.raises(ValueError, match="GPU"):  # everything else is checked, then the device
        T.CacheQuantizer(batch, [1, 1]).write(torch.zeros(2, 2, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 128, dtype=torch.bfloat16), cache)
    with pytest.raises(ValueError, match="blocks of 16"):
        T.BlockSelector(batch, 32, 4)(torch.zeros(2, 8, 128, dtype=torch.bfloat16), cache)


def test_reference_against_torch():
    """The tests' own format against torch's e4m3, and rounding at every midpoint."""
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(quant_ref.e4m3(codes), want, equal_nan=True)
    for bits in (8, 4):
        t = quant_ref.numbers(bits)
        mid = (t[:-1] + t[1:]) / 2
        x = np.zeros((len(mid), 128))
        x[:, 0], x[:, 1], x[:, 2] = mid, -mid, t[-1]  # the power is 1 (256 for the format's border)
        c, s = quant_ref.encode(x, bits)
        assert (s[:, 0] == 127).all()
        v = quant_ref.decode(c, s, bits)
        even = np.where(np.arange(len(mid)) % 2 == 0, t[:-1], t[1:])
        assert np.array_equal(v[:, 0], even) and np.array_equal(v[:, 1], -even)
