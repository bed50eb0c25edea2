"""The quantised cache on the GPU: rows in and out, bounds, chosen blocks and the decode, against tests/quant_ref.py."""
import numpy as np
import pytest
import torch

import paper_2502_12216_amd as T
from attention_ref import close, slopes
import quant_ref as R

pytestmark = pytest.mark.gpu
D = 128


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows_like(g, n, hkv, wild=False):
    """bf16 [n][hkv][128]; wild: groups of every magnitude, zeros, and values at the formats' borders."""
    x = torch.randn(n, hkv, 4, 32, generator=g, device="cuda")
    if wild:
        x = x * torch.exp2(torch.randint(-140, 126, (n, hkv, 4, 1), generator=g, device="cuda").float())
        x = torch.where(torch.rand(n, hkv, 4, 1, generator=g, device="cuda") < 0.1, 0.0, x)
        top = torch.tensor([448.0, 449.0, 464.0, 6.0, 6.03125, 2.0 ** -9, 3.3895313892515355e38, 1.0], device="cuda")
        pick = torch.randint(0, len(top), (n, hkv, 4, 1), generator=g, device="cuda")
        x = torch.where(torch.rand(n, hkv, 4, 1, generator=g, device="cuda") < 0.2, top[pick].expand(-1, -1, -1, 32) *
                        torch.randint(-1, 2, x.shape, generator=g, device="cuda"), x)
    return x.flatten(2).to(torch.bfloat16)


class Held:
    """A quantised cache in spans (page 0) or pages, filled with bytes that mean nothing, and its places."""

    def __init__(self, lens, caps, hq, hkv, bits, page=0, block=0, seed=0):
        self.lens, self.caps, self.hq, self.hkv, self.bits, self.page, self.block = lens, caps, hq, hkv, bits, page, block
        self.batch = T.RaggedBatch(lens, hq, hkv, capacities=caps)
        table = None
        if page:
            counts = [max(1, -(-c // page)) for c in caps]
            order = np.random.default_rng(seed).permutation(sum(counts) + 3).astype(np.int32)
            t = np.zeros((len(lens), max(counts)), np.int32)
            at = 0
            for b, c in enumerate(counts):
                t[b, :c] = order[at:at + c]
                at += c
            table = torch.as_tensor(t, device="cuda")
            self.cache = T.QuantizedCache.empty_pages(self.batch, bits, len(order), page, table, block)
        else:
            self.cache = T.QuantizedCache.empty(self.batch, bits, block)
        g = gen(seed + 99)
        for x in (self.cache.K, self.cache.V, self.cache.K_scale, self.cache.V_scale):
            x.copy_(torch.randint(0, 256, x.shape, generator=g, device="cuda", dtype=torch.uint8))
        if block:
            self.cache.bounds.fill_(float("nan"))

    def at(self, x, b, g, rows):
        """Rows of an array of the cache, numpy."""
        rows = torch.as_tensor(rows, device="cuda").long()
        if not self.page:
            return x[g, int(self.batch.kv_indptr_host[b]) + rows].cpu().numpy()
        page = self.cache.page_table[b].long()[rows // self.page]
        return x[page, g, rows % self.page].cpu().numpy()

    def values(self, name, b, g, rows):
        scale = getattr(self.cache, name + "_scale")
        return R.decode(self.at(getattr(self.cache, name), b, g, rows), self.at(scale, b, g, rows), self.bits)

    def first_block(self, b):
        return int(self.batch.kv_indptr_host[b]) // self.block + b

    def fill(self, seed=1):
        """All rows of every sequence, written as prompts."""
        g = gen(seed)
        n = sum(self.lens)
        k, v = rows_like(g, n, self.hkv), rows_like(g, n, self.hkv)
        T.CacheQuantizer(self.batch, self.lens).write(k, v, self.cache)
        return k, v


LENS = [300, 0, 1, 77, 513, 128]


@pytest.mark.parametrize("wild", [False, True])
@pytest.mark.parametrize("page", [0, 1, 16, 50])
@pytest.mark.parametrize("block", [0, 16, 32, 64, 128])
@pytest.mark.parametrize("bits", [8, 4])
def test_rows_in_and_out(bits, block, page, wild):
    h = Held(LENS, [n + 5 for n in LENS], 4, 2, bits, page, block)
    new = [300, 2, 1, 20, 1, 128]  # a prompt, rows ahead of an empty sequence, chunks, a token, a prompt
    g = gen(5)
    had = [max(0, n - m) for n, m in zip(LENS, new)]
    # what was there before: the rows ahead of the new ones, written as prompts of shorter sequences
    h.batch.seq_len.copy_(torch.tensor(had))
    k0, v0 = rows_like(g, sum(had), 2, wild), rows_like(g, sum(had), 2, wild)
    T.CacheQuantizer(h.batch, had).write(k0, v0, h.cache)
    h.batch.seq_len.copy_(torch.tensor(LENS))
    before = {x: getattr(h.cache, x).clone() for x in ("K", "V", "K_scale", "V_scale")}
    k, v = rows_like(g, sum(new), 2, wild), rows_like(g, sum(new), 2, wild)
    rows = T.CacheQuantizer(h.batch, new)
    rows.write(k, v, h.cache)
    K, V = rows.read(h.cache)
    full = T.CacheQuantizer(h.batch, [n + 3 for n in LENS])
    Ka, Va = full.read(h.cache)
    at, at0, ata = 0, 0, 0
    for b, (n, m) in enumerate(zip(LENS, new)):
        out = max(0, m - n)  # rows ahead of the sequence
        for g_ in range(2):
            for name, x, x0, got, got_all in (("K", k, k0, K, Ka), ("V", v, v0, V, Va)):
                want = torch.cat([x0[at0:at0 + had[b], g_], x[at + out:at + m, g_]]).double().cpu().numpy()
                codes, scales = R.encode(want, bits)
                r = np.arange(n)
                assert np.array_equal(h.at(getattr(h.cache, name), b, g_, r), codes), (b, g_, name)
                assert np.array_equal(h.at(getattr(h.cache, name + "_scale"), b, g_, r), scales), (b, g_, name)
                held = R.decode(codes, scales, bits)
                assert np.array_equal(got[g_, at + out:at + m].double().cpu().numpy(), held[n - (m - out):])
                assert not got[g_, at:at + out].any()
                assert np.array_equal(got_all[g_, ata + 3:ata + 3 + n].double().cpu().numpy(), held)
                assert not got_all[g_, ata:ata + 3].any()
            if block:
                # blocks that no new row touched keep the bounds they had: those of their rows
                ref = R.bounds_of(h.values("K", b, g_, np.arange(n)), block)
                f = h.first_block(b)
                assert np.array_equal(h.cache.bounds[g_, f:f + len(ref)].double().cpu().numpy(), ref), (b, g_)
        # spare rows are as they were
        spare = np.arange(n, h.caps[b])
        for name, old in before.items():
            for g_ in range(2):
                assert np.array_equal(h.at(getattr(h.cache, name), b, g_, spare), h.at(old, b, g_, spare))
        at, at0, ata = at + m, at0 + had[b], ata + n + 3
    if block:  # places of no block are as they were
        used = torch.zeros(h.cache.bounds.shape[1], dtype=torch.bool)
        for b, n in enumerate(LENS):
            used[h.first_block(b):h.first_block(b) + -(-n // block)] = True
        assert torch.isnan(h.cache.bounds[:, ~used.cuda()].float()).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_groups_that_are_not_finite(bits):
    h = Held([70], [70], 4, 2, bits, block=32)
    g = gen(3)
    k, v = rows_like(g, 70, 2), rows_like(g, 70, 2)
    k[5, 0, 40], k[33, 1, 0], v[69, 0, 127], v[2, 1, 64] = float("nan"), float("inf"), -float("inf"), float("nan")
    rows = T.CacheQuantizer(h.batch, [70])
    rows.write(k, v, h.cache)
    K, V = rows.read(h.cache)
    for got, x in ((K, k), (V, v)):
        ref = np.stack([R.decode(*R.encode(x[:, j].double().cpu().numpy(), bits), bits) for j in range(2)])
        assert np.isnan(ref).sum() == 64
        assert np.array_equal(got.double().cpu().numpy(), ref, equal_nan=True)
    for j in range(2):
        ref = R.bounds_of(h.values("K", 0, j, np.arange(70)), 32)
        assert np.array_equal(h.cache.bounds[j, :3].double().cpu().numpy(), ref, equal_nan=True)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("bits", [8, 4])
def test_token_by_token_is_as_the_prompt(bits, block):
    n = 140
    a, c = Held([n], [n], 4, 2, bits, block=block), Held([0], [n], 4, 2, bits, block=block)
    k, v = a.fill()
    one = T.CacheQuantizer(c.batch, [1])
    for i in range(n):
        c.batch.seq_len += 1
        one.write(k[i:i + 1], v[i:i + 1], c.cache)
    for x in ("K", "V", "K_scale", "V_scale"):
        assert torch.equal(getattr(a.cache, x), getattr(c.cache, x))
    nb = -(-n // block)
    assert torch.equal(a.cache.bounds[:, :nb], c.cache.bounds[:, :nb])


def check_decode(h, q, out, lse, chosen=None, cap=0.0, sl=None):
    """out and lse of every head against 64 bits; chosen[b][g]: the blocks attended (None: all rows)."""
    G = h.hq // h.hkv
    for b, n in enumerate(h.lens):
        for g in range(h.hkv):
            rows = np.arange(n) if chosen is None else R.rows_of_blocks(chosen[b][g], h.block, n)
            k, v = (torch.as_tensor(h.values(x, b, g, rows), device="cuda") for x in ("K", "V"))
            for j in range(g * G, g * G + G):
                if len(rows) == 0:
                    assert not out[b, j].any() and lse[b, j] == -np.inf
                    continue
                o, l, _, mean_abs, off = R.one_token(q[b, j], k, v, rows, n, cap, 0.0 if sl is None else float(sl[j]))
                close(out[b, j][None], o, R.tolerance(mean_abs, off, o, len(rows)), f"out {b} {j}")
                close(lse[b, j][None], l, R.tolerance_lse(off, l, len(rows)), f"lse {b} {j}")


@pytest.mark.parametrize("mod", [(0.0, False), (50.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("page", [0, 1, 16, 50])
@pytest.mark.parametrize("hq,hkv", [(3, 3), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("bits", [8, 4])
def test_decode(bits, hq, hkv, page, mod):
    lens = [0, 1, 5, 33, 129, 1000, 2501]
    h = Held(lens, [n + 9 for n in lens], hq, hkv, bits, page)
    h.fill()
    q = (2 * torch.randn(len(lens), hq, D, generator=gen(7), device="cuda")).to(torch.bfloat16)
    sl = slopes(hq) if mod[1] else None
    out, lse = T.QuantizedDecoder(h.batch)(q, h.cache, T.ScoreMod(cap=mod[0], slopes=sl))
    check_decode(h, q, out, lse, cap=mod[0], sl=sl)


@pytest.mark.parametrize("hq", [1, 8])
@pytest.mark.parametrize("bits", [8, 4])
def test_decode_rising_scores(bits, hq):
    """Scores that rise by more than the reference's slack along the cache, and ones that fall."""
    n = 3000
    h = Held([n, n], [n, n], hq, 1, bits)
    k, v = rows_like(gen(1), 2 * n, 1), rows_like(gen(2), 2 * n, 1)
    ramp = torch.linspace(-30, 30, n, device="cuda")
    k += (torch.cat([ramp, -ramp])[:, None, None] / 4).to(torch.bfloat16)
    T.CacheQuantizer(h.batch, h.lens).write(k, v, h.cache)
    q = torch.full((2, hq, D), 1.0, dtype=torch.bfloat16, device="cuda")
    out, lse = T.QuantizedDecoder(h.batch)(q, h.cache)
    check_decode(h, q, out, lse)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("bits", [8, 4])
def test_nan_reaches_the_heads_that_see_it(bits, page):
    h = Held([400, 300], [405, 305], 8, 2, bits, page)
    g = gen(4)
    k, v = rows_like(g, 700, 2), rows_like(g, 700, 2)
    k[399, 0, 3] = float("nan")       # sequence 0, KV head 0: every head of it
    v[400, 1, 100] = float("inf")     # sequence 1, KV head 1: dimensions 96 .. 127
    k[400, 1] = -200                  # at a weight of 0
    T.CacheQuantizer(h.batch, h.lens).write(k, v, h.cache)
    q = torch.ones(2, 8, D, dtype=torch.bfloat16, device="cuda")
    out, lse = T.QuantizedDecoder(h.batch)(q, h.cache)
    nan = torch.zeros(2, 8, D, dtype=torch.bool, device="cuda")
    nan[0, :4] = True
    nan[1, 4:, 96:] = True
    assert torch.equal(torch.isnan(out), nan)
    assert torch.isnan(lse[0, :4]).all() and torch.isfinite(lse[0, 4:]).all() and torch.isfinite(lse[1]).all()


def choices(h, q, budget, first, last):
    G = h.hq // h.hkv
    got = []
    for b, n in enumerate(h.lens):
        nb, f = -(-n // h.block), h.first_block(b)
        got.append([R.choose(q[b, g * G:g * G + G].double().cpu().numpy(), h.cache.bounds[g, f:f + nb].double().cpu().numpy(),
                             budget, first, last) for g in range(h.hkv)])
    return got


def check_choice(want, blocks, counts):
    for b, per in enumerate(want):
        for g, w in enumerate(per):
            assert int(counts[b, g]) == len(w)
            row = blocks[b, g].cpu().numpy()
            assert np.array_equal(row[:len(w)], w), (b, g)
            assert (row[len(w):] == -1).all()


@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (1, 0, 1), (5, 1, 2), (12, 4, 8), (40, 0, 1), (1000, 1, 2)])
@pytest.mark.parametrize("hq,hkv", [(3, 3), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("block,page", [(16, 0), (32, 50), (64, 16), (128, 0)])
def test_choice_and_decode_of_blocks(block, page, hq, hkv, budget, first, last):
    lens = [0, 1, 17, 600, 2049, 128 * 20]
    h = Held(lens, [n + 9 for n in lens], hq, hkv, 8 if block > 16 else 4, page, block)
    h.fill()
    q = (2 * torch.randn(len(lens), hq, D, generator=gen(7), device="cuda")).to(torch.bfloat16)
    blocks, counts = T.BlockSelector(h.batch, block, budget, first, last)(q, h.cache)
    want = choices(h, q, budget, first, last)
    check_choice(want, blocks, counts)
    sl = slopes(hq)
    dec = T.QuantizedDecoder(h.batch)
    out, lse = dec(q, h.cache, blocks=blocks, counts=counts)
    check_decode(h, q, out, lse, want)
    out, lse = dec(q, h.cache, T.ScoreMod(cap=20.0, slopes=sl), blocks=blocks, counts=counts)
    check_decode(h, q, out, lse, want, cap=20.0, sl=sl)


def only_bounds(nb, block, hq, hkv, seed=0):
    """A cache of which only the bounds matter, and its batch."""
    batch = T.RaggedBatch([nb * block - 3], hq, hkv, capacities=[nb * block])
    c = torch.zeros(hkv, 1, 128, dtype=torch.uint8, device="cuda")
    s = torch.zeros(hkv, 1, 4, dtype=torch.uint8, device="cuda")
    x = torch.randn(hkv, nb + 1, 2, D, generator=gen(seed), device="cuda").sort(2).values.to(torch.bfloat16)
    return batch, T.QuantizedCache(c, s, c, s, bounds=x, block=block)


@pytest.mark.parametrize("nb", [1000, 1025, 2048, 4000, 8192, 16384, 16385, 40001])
def test_choice_of_many_blocks(nb):
    """Every number of blocks per thread, and keys in the workspace."""
    batch, cache = only_bounds(nb, 16, 8, 2)
    q = torch.randn(1, 8, D, generator=gen(1), device="cuda").to(torch.bfloat16)
    for budget in (1, 100, nb - 1):
        blocks, counts = T.BlockSelector(batch, 16, budget, 0, 1)(q, cache)
        for g in range(2):
            want = R.choose(q[0, 4 * g:4 * g + 4].double().cpu().numpy(), cache.bounds[g, :nb].double().cpu().numpy(), budget, 0, 1)
            assert int(counts[0, g]) == budget and np.array_equal(blocks[0, g].cpu().numpy(), want)


@pytest.mark.parametrize("nb", [30, 150, 300, 3000, 20000])
def test_choice_among_equals(nb):
    """Ties go to the lower block: a query of zeros, three kinds of blocks, and bounds of NaN above all."""
    batch, cache = only_bounds(nb, 16, 4, 1)
    q = torch.zeros(1, 4, D, dtype=torch.bfloat16, device="cuda")
    budget = nb // 3
    blocks, _ = T.BlockSelector(batch, 16, budget, 0, 0)(q, cache)
    assert np.array_equal(blocks[0, 0].cpu().numpy(), np.arange(budget))
    cache.bounds.copy_(cache.bounds[:, torch.arange(nb + 1) % 3])
    cache.bounds[0, [nb // 2, nb - 2], 1, 7] = float("nan")
    q = torch.randn(1, 4, D, generator=gen(1), device="cuda").to(torch.bfloat16)
    q[0, :, 7] = 1.0
    blocks, _ = T.BlockSelector(batch, 16, budget, 2, 1)(q, cache)
    want = R.choose(q[0].double().cpu().numpy(), cache.bounds[0, :nb].double().cpu().numpy(), budget, 2, 1)
    assert nb // 2 in want and nb - 2 in want
    assert np.array_equal(blocks[0, 0].cpu().numpy(), want)


@pytest.mark.parametrize("size", [1e-30, 1.0, 3e38])
@pytest.mark.parametrize("nb", [100, 300, 3000, 20000])
def test_choice_of_any_size_beside_infinities(nb, size):
    """Scores in the type's highest and lowest reaches, with one head's best infinite: its block above all."""
    batch, cache = only_bounds(nb, 16, 2, 1)
    cache.bounds.zero_()
    cache.bounds[0, :nb, :, 0] = (-size * torch.rand(nb, 1, generator=gen(3), device="cuda")).to(torch.bfloat16)
    cache.bounds[0, nb // 2, 1, 1] = float("inf")
    q = torch.zeros(1, 2, D, dtype=torch.bfloat16, device="cuda")
    q[0, 0, 0], q[0, 1, 1] = 1.0, 1.0
    budget = nb // 4
    with np.errstate(invalid="ignore"):
        want = R.choose(q[0].double().cpu().numpy(), cache.bounds[0, :nb].double().cpu().numpy(), budget, 0, 0)
    assert nb // 2 in want
    blocks, _ = T.BlockSelector(batch, 16, budget, 0, 0)(q, cache)
    assert np.array_equal(blocks[0, 0].cpu().numpy(), want)


@pytest.mark.parametrize("hq", [1, 2, 4, 8])
@pytest.mark.parametrize("nb", [60, 700])
def test_choice_with_bounds_far_apart(hq, nb):
    """The bound that a query's sign leaves out does not touch the score, however large it is."""
    budget = nb // 10
    batch, cache = only_bounds(nb, 16, hq, 1)
    x = torch.randn(nb, D, generator=gen(4), device="cuda")
    far = 3e38 * torch.rand(nb, D, generator=gen(5), device="cuda") + 1e30
    even = torch.arange(D, device="cuda") % 2 == 0
    cache.bounds[0, :nb, 0] = torch.where(even, -far, x).to(torch.bfloat16)
    cache.bounds[0, :nb, 1] = torch.where(even, x, far).to(torch.bfloat16)
    q = torch.randn(1, hq, D, generator=gen(6), device="cuda").abs()
    q = torch.where(even, q, -q).to(torch.bfloat16)
    want = R.choose(q[0].double().cpu().numpy(), cache.bounds[0, :nb].double().cpu().numpy(), budget, 0, 0)
    blocks, _ = T.BlockSelector(batch, 16, budget, 0, 0)(q, cache)
    assert np.array_equal(blocks[0, 0].cpu().numpy(), want)


def test_decode_of_all_blocks_is_the_decode():
    lens = [700, 33]
    h = Held(lens, [n + 9 for n in lens], 8, 2, 8, block=32)
    h.fill()
    q = torch.randn(2, 8, D, generator=gen(7), device="cuda").to(torch.bfloat16)
    dec = T.QuantizedDecoder(h.batch)
    blocks, counts = T.BlockSelector(h.batch, 32, 22)(q, h.cache)
    a = [x.clone() for x in dec(q, h.cache)]
    c = dec(q, h.cache, blocks=blocks, counts=counts)
    assert all(torch.equal(x, y) for x, y in zip(a, c))


@pytest.mark.parametrize("bits", [8, 4])
def test_cache_past_2_31_bytes(bits):
    """The last rows of arrays of more than 2^31 bytes: a short sequence behind a long one."""
    n = (2 ** 31 // (16 * bits * 2)) + 1000
    h = Held([3, 900], [n, 905], 8, 2, bits, block=64)
    assert h.cache.K.numel() > 2 ** 31
    h.fill()
    q = torch.randn(2, 8, D, generator=gen(7), device="cuda").to(torch.bfloat16)
    out, lse = T.QuantizedDecoder(h.batch)(q, h.cache)
    check_decode(h, q, out, lse)
    blocks, counts = T.BlockSelector(h.batch, 64, 5)(q, h.cache)
    check_choice(choices(h, q, 5, 1, 2), blocks, counts)
    h.batch.seq_len[0] = n  # the long one's rows: a read of its last ones
    rows = T.CacheQuantizer(h.batch, [5, 2])
    k = rows_like(gen(9), 7, 2)
    rows.write(k, k, h.cache)
    K, V = rows.read(h.cache)
    ref = np.stack([R.decode(*R.encode(k[:, j].double().cpu().numpy(), bits), bits) for j in range(2)])
    assert np.array_equal(K.double().cpu().numpy(), ref) and torch.equal(K, V)


@pytest.mark.parametrize("longest", [40, 2100])
@pytest.mark.parametrize("blocks", [False, True])
def test_as_many_groups_as_there_may_be(longest, blocks):
    """512 sequences of 8 KV heads, most of a few rows or none: by one workgroup each, and split."""
    lens = [longest] + [i % 6 for i in range(511)]
    h = Held(lens, lens, 64, 8, 8, block=16)
    h.fill()
    q = torch.randn(512, 64, D, generator=gen(3), device="cuda").to(torch.bfloat16)
    dec, sel = T.QuantizedDecoder(h.batch), T.BlockSelector(h.batch, 16, 131, 0, 1)
    b, c = sel(q, h.cache)
    out, lse = dec(q, h.cache, blocks=b, counts=c) if blocks else dec(q, h.cache)
    few = [0, 1, 2, 3, 4, 5, 6, 511]
    assert not out[[i for i, n in enumerate(lens) if n == 0]].any()
    sub = Held([lens[i] for i in few], [lens[i] for i in few], 64, 8, 8, block=16)
    for at, i in enumerate(few):  # the same rows in a cache of their own
        a, z, n = int(h.batch.kv_indptr_host[i]), int(sub.batch.kv_indptr_host[at]), lens[i]
        for x in ("K", "V", "K_scale", "V_scale"):
            getattr(sub.cache, x)[:, z:z + n] = getattr(h.cache, x)[:, a:a + n]
        if lens[i]:
            f = h.first_block(i)
            sub.cache.bounds[:, sub.first_block(at):sub.first_block(at) + -(-n // 16)] = h.cache.bounds[:, f:f + -(-n // 16)]
    want = choices(sub, q[few], 131, 0, 1)  # (132 blocks of the long one)
    check_choice(want, b[few], c[few])
    check_decode(sub, q[few], out[few], lse[few], want if blocks else None)


@pytest.mark.parametrize("page", [0, 16])
def test_spans_without_spare_rows(page):
    """No device lengths: every span is full."""
    lens = [130, 1, 64]
    h = Held(lens, lens, 8, 2, 8, page, 32)
    full = T.RaggedBatch(lens, 8, 2)
    assert full.seq_len is None
    g = gen(1)
    k, v = rows_like(g, 195, 2), rows_like(g, 195, 2)
    rows = T.CacheQuantizer(full, lens)
    rows.write(k, v, h.cache)
    got = [x.clone() for x in rows.read(h.cache)]
    assert all(torch.equal(x, y) for x, y in zip(got, T.CacheQuantizer(h.batch, lens).read(h.cache)))
    q = torch.randn(3, 8, D, generator=g, device="cuda").to(torch.bfloat16)
    b, c = T.BlockSelector(full, 32, 3)(q, h.cache)
    want = choices(h, q, 3, 1, 2)
    check_choice(want, b, c)
    out, lse = T.QuantizedDecoder(full)(q, h.cache, blocks=b, counts=c)
    check_decode(h, q, out, lse, want)


def test_empty_chunks_and_refused_ones():
    c = T.QuantizingCache(4, 2, [40, 40], bits=8, block=32)
    def some(m, heads, dtype=torch.bfloat16):
        return torch.randn(m, heads, D, generator=gen(m + heads), device="cuda").to(dtype)
    assert c.extend([some(0, 4)] * 2, [some(0, 2)] * 2, [some(0, 2)] * 2).shape == (0, 4, D)
    assert c.batch.seq_lens == [0, 0] and not c.decode(some(2, 4)).any()
    for bad in (([some(3, 4)] * 2, [some(3, 2)] * 2, [some(2, 2)] * 2), ([some(3, 4)], [some(3, 2)], [some(3, 2)]),
                ([some(3, 4)] * 2, [some(3, 2, torch.float32)] * 2, [some(3, 2)] * 2),
                ([some(3, 2)] * 2, [some(3, 2)] * 2, [some(3, 2)] * 2)):
        with pytest.raises((TypeError, ValueError)):
            c.extend(*bad)
    assert c.batch.seq_lens == [0, 0] and c.batch.seq_len.tolist() == [0, 0]
    assert c.extend([some(3, 4), some(0, 4)], [some(3, 2), some(0, 2)], [some(3, 2), some(0, 2)]).shape == (3, 4, D)
    assert c.batch.seq_len.tolist() == [3, 0]


def test_captured_steps_and_streams():
    """A step (length, write, choice, decode) captured, replayed with eager work between, on another stream, and beside a
    second captured step of the same objects."""
    lens, hq, hkv, steps = [200, 64, 0], 8, 2, 5
    h = Held(lens, [n + 40 for n in lens], hq, hkv, 8, block=32)
    e = Held(lens, [n + 40 for n in lens], hq, hkv, 8, block=32)
    for x in (h, e):
        x.fill()
    g = gen(11)
    ks, vs = (torch.randn(2 * steps, 3, hkv, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    qs = torch.randn(2 * steps, 3, hq, D, generator=g, device="cuda").to(torch.bfloat16)

    def parts(x):
        return T.CacheQuantizer(x.batch, [1, 1, 1]), T.BlockSelector(x.batch, 32, 4), T.QuantizedDecoder(x.batch)

    def step(x, p, k, v, q):
        x.batch.seq_len += 1
        p[0].write(k, v, x.cache)
        b, c = p[1](q, x.cache)
        return p[2](q, x.cache, blocks=b, counts=c)

    ph, pe = parts(h), parts(e)
    k, v, q = ks[0].clone(), vs[0].clone(), qs[0].clone()
    out = torch.empty(3, hq, D, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(s):
        keep = [x.clone() for x in (h.batch.seq_len, h.cache.K, h.cache.V, h.cache.K_scale, h.cache.V_scale, h.cache.bounds)]
        step(h, ph, k, v, q)
        for x, y in zip((h.batch.seq_len, h.cache.K, h.cache.V, h.cache.K_scale, h.cache.V_scale, h.cache.bounds), keep):
            x.copy_(y)
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                out.copy_(step(h, ph, k, v, q)[0])
            graphs.append(graph)
        for i in range(2 * steps):
            k.copy_(ks[i])
            v.copy_(vs[i])
            q.copy_(qs[i])
            graphs[i % 2].replay()
            want, _ = step(e, pe, ks[i], vs[i], qs[i])
            s.synchronize()
            assert torch.equal(out, want), i
    for x in ("K", "V", "K_scale", "V_scale"):
        for b, n in enumerate(lens):
            a, z = int(h.batch.kv_indptr_host[b]), int(h.batch.kv_indptr_host[b]) + n + 2 * steps
            assert torch.equal(getattr(h.cache, x)[:, a:z], getattr(e.cache, x)[:, a:z])


@pytest.mark.parametrize("budget", [0, 6])
@pytest.mark.parametrize("bits", [8, 4])
def test_quantizing_cache(bits, budget):
    """Prompts in two chunks, then tokens: attention over what the cache holds."""
    hq, hkv, caps = 8, 2, [500, 300, 64]
    c = T.QuantizingCache(hq, hkv, caps, bits=bits, block=32, budget=budget)
    g = gen(21)

    def some(m, heads):
        return torch.randn(m, heads, D, generator=g, device="cuda").to(torch.bfloat16)

    held = [[] for _ in caps]
    for new in ([300, 10, 0], [150, 200, 3]):
        q, K, V = ([some(m, x) for m in new] for x in (hq, hkv, hkv))
        out = c.extend(q, K, V)
        assert out.shape == (sum(new), hq, D)
        for b in range(3):
            held[b].append((K[b], V[b]))
    lens = [450, 210, 3]
    for i in range(4):
        k, v, q = some(3, hkv), some(3, hkv), some(3, hq)
        c.append(k, v)
        got = c.decode(q)
        for b in range(3):
            held[b].append((k[b:b + 1], v[b:b + 1]))
        lens = [n + 1 for n in lens]
        assert c.batch.seq_lens == lens and c.batch.seq_len.tolist() == lens
        for b, n in enumerate(lens):
            K, V = (torch.cat([x[j] for x in held[b]]) for j in (0, 1))
            for gg in range(hkv):
                kv = [R.decode(*R.encode(x[:, gg].double().cpu().numpy(), bits), bits) for x in (K, V)]
                rows = np.arange(n)
                if budget:
                    rows = R.rows_of_blocks(R.choose(q[b, 4 * gg:4 * gg + 4].double().cpu().numpy(), R.bounds_of(kv[0], 32), budget, 1, 2), 32, n)
                kk, vv = (torch.as_tensor(x[rows], device="cuda") for x in kv)
                for j in range(4 * gg, 4 * gg + 4):
                    o, _, _, mean_abs, off = R.one_token(q[b, j], kk, vv, rows, n)
                    close(got[b, j][None], o, R.tolerance(mean_abs, off, o, n), f"{i} {b} {j}")
    with pytest.raises(ValueError, match="outgrew"):
        c.extend([some(m, hq) for m in (60, 0, 0)], [some(m, hkv) for m in (60, 0, 0)], [some(m, hkv) for m in (60, 0, 0)])
    with pytest.raises((TypeError, ValueError)):
        c.append(k.float(), v)
    assert c.batch.seq_len.tolist() == lens


@pytest.mark.parametrize("fails", ["slopes", "cache", "memory", "attention"])
def test_extend_that_fails_counts_nothing(fails, monkeypatch):
    """The lengths stay those of before, and the same chunk again gives what it gives a cache without a failure."""
    import paper_2502_12216_amd.cache as module
    sl, g = slopes(4), gen(31)

    def some(heads):
        return [torch.randn(m, heads, D, generator=g, device="cuda").to(torch.bfloat16) for m in (40, 7)]

    first, chunk = ([some(4), some(2), some(2)] for _ in range(2))
    c, e = (T.QuantizingCache(4, 2, [100, 100], bits=8, block=32, slopes=sl) for _ in range(2))
    c.extend(*first)
    e.extend(*first)
    before = [getattr(c.cache, x).clone() for x in ("K", "K_scale", "V", "V_scale", "bounds")]

    def no_memory(*args, **kw):
        raise torch.OutOfMemoryError("no memory")

    with monkeypatch.context() as mp:
        if fails == "slopes":
            mp.setattr(c, "mod", T.ScoreMod(slopes=sl.double()))
        elif fails == "cache":
            mp.setattr(c.cache, "V", c.cache.V[:, :-1].contiguous())
        elif fails == "memory":
            mp.setattr(module, "PromptAttention", no_memory)
        else:
            mp.setattr(module.PromptAttention, "__call__", no_memory)
        with pytest.raises((TypeError, ValueError, torch.OutOfMemoryError)):
            c.extend(*chunk)
    assert c.batch.seq_lens == [40, 7] and c.batch.seq_len.tolist() == [40, 7]
    if fails != "attention":  # (refused before anything was written)
        assert all(torch.equal(getattr(c.cache, x), y) for x, y in zip(("K", "K_scale", "V", "V_scale", "bounds"), before))
    assert torch.equal(c.extend(*chunk), e.extend(*chunk))
    assert c.batch.seq_len.tolist() == [80, 14]
    for x in ("K", "K_scale", "V", "V_scale", "bounds"):
        assert torch.equal(getattr(c.cache, x), getattr(e.cache, x))


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("bits", [8, 4])
def test_rows_of_pages_that_are_not_there(bits, block):
    """Table entries of -1, num_pages and beyond: their rows are not written, read as zeros and count as zeros in the
    bounds, new rows as those from before; other pages are as they would be without them."""
    n, page, hkv = 200, 16, 2
    h, full = Held([n], [n], 4, hkv, bits, page, block), Held([n], [n], 4, hkv, bits, page, block)
    num = h.cache.K.shape[0]
    gone = {1: -1, 4: num, 9: num + 1000, 12: -2 ** 31}
    for i, entry in gone.items():
        h.cache.page_table[0, i] = entry
    missing = np.isin(np.arange(n) // page, list(gone))
    k, v = rows_like(gen(1), n, hkv), rows_like(gen(2), n, hkv)
    k[:, :, 0] += 4.0   # a dimension whose least value is a missing row's zero
    k[page, 0, 40] = float("nan")  # of a row that is not written
    for x in (h, full):
        for m in (75, 1, 124):  # a chunk, a token, the rest, from inside a missing page
            x.batch.seq_len[0] = {75: 75, 1: 76, 124: n}[m]
            at = slice(int(x.batch.seq_len[0]) - m, int(x.batch.seq_len[0]))
            T.CacheQuantizer(x.batch, [m]).write(k[at].contiguous(), v[at].contiguous(), x.cache)
    K, V = T.CacheQuantizer(h.batch, [n]).read(h.cache)
    for name, got in (("K", K), ("V", V)):
        for g in range(hkv):
            held = full.values(name, 0, g, np.arange(n))
            held[missing] = 0.0
            assert np.array_equal(got[g].double().cpu().numpy(), held)
            if name == "K":
                ref = R.bounds_of(held, block)
                assert np.array_equal(h.cache.bounds[g, :len(ref)].double().cpu().numpy(), ref), g
    for name in ("K", "V", "K_scale", "V_scale"):  # only the pages that are there were written
        x, y, fresh = (getattr(z.cache, name) for z in (h, full, Held([n], [n], 4, hkv, bits, page, block)))
        ids = full.cache.page_table[0].long()
        there = torch.tensor([i not in gone for i in range(len(ids))], device="cuda")
        assert torch.equal(x[ids[there]], y[ids[there]])
        other = torch.ones(num, dtype=torch.bool, device="cuda")
        other[ids[there]] = False
        assert torch.equal(x[other], fresh[other])


@pytest.mark.parametrize("page", [0, 16, 50])
@pytest.mark.parametrize("bits", [8, 4])
def test_powers_at_any_word(bits, page):
    """K_scale and V_scale need 4-byte alignment only, and sequences of spans begin at any row."""
    lens = [2500, 33, 130, 7, 300]
    a, c = (Held(lens, [n + 1 for n in lens], 8, 2, bits, page, 32) for _ in range(2))
    for i, x in enumerate(("K_scale", "V_scale")):
        old = getattr(c.cache, x)
        room = torch.empty(old.numel() + 16, dtype=torch.uint8, device="cuda")
        moved = room[4 + 4 * i:4 + 4 * i + old.numel()].view(old.shape)
        assert moved.data_ptr() % 16 == 4 + 4 * i
        setattr(c.cache, x, moved.copy_(old))
    q = torch.randn(len(lens), 8, D, generator=gen(7), device="cuda").to(torch.bfloat16)
    got = []
    for h in (a, c):
        h.fill()
        got.append(T.CacheQuantizer(h.batch, lens).read(h.cache) + T.QuantizedDecoder(h.batch)(q, h.cache))
        assert torch.equal(h.cache.V_scale, a.cache.V_scale) and torch.equal(h.cache.K_scale, a.cache.K_scale)
    assert all(torch.equal(x, y) for x, y in zip(*got))
    check_decode(c, q, got[1][2], got[1][3])
