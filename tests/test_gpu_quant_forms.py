"""Every form of the quantised decode and of the block choice that the sizes of a call select: the decode by one workgroup
for each KV head, the choice by the workgroup that scores, on both sides of their limits; every bf16 value in and out."""
import numpy as np
import pytest
import torch

import paper_2502_12216_amd as T
from attention_ref import slopes
import quant_ref as R
from test_gpu_quant import D, Held, check_choice, check_decode, choices, gen, rows_like

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mod", [(0.0, False), (50.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("page", [0, 1, 16, 50])
@pytest.mark.parametrize("hq,hkv", [(3, 3), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("bits", [8, 4])
def test_decode_of_short_spans(bits, hq, hkv, page, mod):
    """Spans of at most 309 rows: a workgroup for each KV head."""
    lens = [0, 1, 5, 33, 128, 129, 300]
    h = Held(lens, [n + 9 for n in lens], hq, hkv, bits, page)
    h.fill()
    q = (2 * torch.randn(len(lens), hq, D, generator=gen(7), device="cuda")).to(torch.bfloat16)
    sl = slopes(hq) if mod[1] else None
    out, lse = T.QuantizedDecoder(h.batch)(q, h.cache, T.ScoreMod(cap=mod[0], slopes=sl))
    check_decode(h, q, out, lse, cap=mod[0], sl=sl)


@pytest.mark.parametrize("spare", [0, 3000])
@pytest.mark.parametrize("page", [0, 16, 50])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("bits", [8, 4])
def test_rising_scores_and_lists_by_both_forms(bits, hq, hkv, page, spare):
    """Short sequences whose scores rise past the reference's slack, in short spans and in long ones (which are split),
    all rows and those of chosen blocks, with a cap and slopes."""
    lens = [0, 260, 31, 290]
    h = Held(lens, [n + spare for n in lens], hq, hkv, bits, page, 16)
    total = sum(lens)
    k, v = rows_like(gen(1), total, hkv), rows_like(gen(2), total, hkv)
    ramp = torch.cat([torch.linspace(-20, 20, n, device="cuda") for n in lens if n])
    k += (ramp[:, None, None] / 4).to(torch.bfloat16)
    T.CacheQuantizer(h.batch, lens).write(k, v, h.cache)
    q = torch.randn(len(lens), hq, D, generator=gen(7), device="cuda").abs().to(torch.bfloat16)
    sl, dec = slopes(hq), T.QuantizedDecoder(h.batch)
    check_decode(h, q, *dec(q, h.cache))
    check_decode(h, q, *dec(q, h.cache, T.ScoreMod(cap=30.0, slopes=sl)), cap=30.0, sl=sl)
    blocks, counts = T.BlockSelector(h.batch, 16, 7)(q, h.cache)
    want = choices(h, q, 7, 1, 2)
    check_choice(want, blocks, counts)
    check_decode(h, q, *dec(q, h.cache, T.ScoreMod(cap=30.0, slopes=sl), blocks=blocks, counts=counts), want, cap=30.0, sl=sl)


@pytest.mark.parametrize("spare", [0, 3000])
@pytest.mark.parametrize("bits", [8, 4])
def test_nan_by_both_forms(bits, spare):
    """A key's NaN and a value's infinity at a weight of 0, as in short spans, also where the rows are split."""
    h = Held([400, 300], [400 + spare, 300 + spare], 8, 2, bits)
    k, v = rows_like(gen(4), 700, 2), rows_like(gen(5), 700, 2)
    k[399, 0, 3] = float("nan")
    v[400, 1, 100] = float("inf")
    k[400, 1] = -200
    T.CacheQuantizer(h.batch, h.lens).write(k, v, h.cache)
    q = torch.ones(2, 8, D, dtype=torch.bfloat16, device="cuda")
    out, lse = T.QuantizedDecoder(h.batch)(q, h.cache)
    nan = torch.zeros(2, 8, D, dtype=torch.bool, device="cuda")
    nan[0, :4] = True
    nan[1, 4:, 96:] = True
    assert torch.equal(torch.isnan(out), nan)
    assert torch.isnan(lse[0, :4]).all() and torch.isfinite(lse[0, 4:]).all() and torch.isfinite(lse[1]).all()


@pytest.mark.parametrize("nb", [191, 192, 193, 257, 512, 513, 1000, 1024, 1025])
@pytest.mark.parametrize("hq", [8, 16, 32, 64])
def test_choice_of_256_groups(hq, nb):
    """32 sequences of 8 KV heads, one or a few as long as the longest: scored by the workgroup that selects up to 1024
    blocks (512 with eight heads), by a launch of their own beyond."""
    lens = [(0, 1, 77, 16 * nb // 3, 16 * 40)[b % 5] for b in range(32)]
    lens[3], lens[31] = 16 * nb, 16 * nb - 7
    batch = T.RaggedBatch(lens, hq, 8, capacities=lens)
    assert batch.max_len == 16 * nb
    bounds = torch.randn(8, batch.total // 16 + 32, 2, D, generator=gen(3), device="cuda").sort(2).values.to(torch.bfloat16)
    none = torch.zeros(8, 1, D, dtype=torch.uint8, device="cuda")
    cache = T.QuantizedCache(none, none[..., :4], none, none[..., :4], bounds=bounds, block=16)
    q = torch.randn(32, hq, D, generator=gen(1), device="cuda").to(torch.bfloat16)
    for budget, first, last in ((33, 1, 2), (nb - 1, 0, 0)):
        blocks, counts = T.BlockSelector(batch, 16, budget, first, last)(q, cache)
        for b in (0, 1, 2, 3, 4, 8, 31):
            held = -(-lens[b] // 16)
            f = int(batch.kv_indptr_host[b]) // 16 + b
            for g in (0, 7):
                heads = q[b, g * (hq // 8):(g + 1) * (hq // 8)].double().cpu().numpy()
                want = R.choose(heads, bounds[g, f:f + held].double().cpu().numpy(), budget, first, last)
                assert int(counts[b, g]) == len(want), (b, g, budget)
                row = blocks[b, g].cpu().numpy()
                assert np.array_equal(row[:len(want)], want) and (row[len(want):] == -1).all(), (b, g, budget)


@pytest.mark.parametrize("hq", [1, 2, 4, 8])
@pytest.mark.parametrize("nb", [64, 65, 192, 193, 256, 257])
def test_choice_at_the_limits_of_one_launch(hq, nb):
    """One sequence of one KV head, on both sides of the numbers of blocks up to which the workgroup that selects scores."""
    batch = T.RaggedBatch([16 * nb - 3], hq, 1, capacities=[16 * nb])
    none = torch.zeros(1, 1, D, dtype=torch.uint8, device="cuda")
    bounds = torch.randn(1, nb + 1, 2, D, generator=gen(nb), device="cuda").sort(2).values.to(torch.bfloat16)
    cache = T.QuantizedCache(none, none[..., :4], none, none[..., :4], bounds=bounds, block=16)
    q = torch.randn(1, hq, D, generator=gen(1), device="cuda").to(torch.bfloat16)
    for budget, first, last in ((1, 0, 0), (20, 1, 2), (nb - 1, 0, 1)):
        blocks, counts = T.BlockSelector(batch, 16, budget, first, last)(q, cache)
        want = R.choose(q[0].double().cpu().numpy(), bounds[0, :nb].double().cpu().numpy(), budget, first, last)
        assert int(counts[0, 0]) == budget and np.array_equal(blocks[0, 0].cpu().numpy(), want)


@pytest.mark.parametrize("bits", [8, 4])
def test_every_bf16_value(bits):
    """Each of the 65536 bf16 values beside every largest value that changes a power or lies at a border of its range: codes,
    powers, bounds and the values read back."""
    x = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    finite = torch.isfinite(x)
    values = torch.cat([torch.nn.functional.pad(part, (0, -len(part) % 31)) for part in (x[finite], x[~finite])]).view(-1, 31)
    n = len(values)
    # a group's largest: a full group, just past one, the borders of the powers' range, the least and largest bf16
    most = 1.75 if bits == 8 else 1.5
    tops = [0.0] + [m * 2.0 ** e for e in (-126, -110, -109, -108, 0, 8, 100, 126, 127) for m in (1.0, most, most + 2.0 ** -7)]
    tops = torch.tensor(tops, device="cuda", dtype=torch.float64).to(torch.bfloat16)
    h = Held([n], [n], 1, 1, bits, block=16)
    rows = T.CacheQuantizer(h.batch, [n])
    for some in tops.split(4):  # one for each group of the row
        row = torch.zeros(n, 1, 4, 32, dtype=torch.bfloat16, device="cuda")
        row[:, 0, :, :31] = values[:, None]
        for i, top in enumerate(some):
            row[:, 0, i, 31] = -top
        k = row.flatten(2)
        rows.write(k, k, h.cache)
        K, V = rows.read(h.cache)
        codes, scales = R.encode(k[:, 0].double().cpu().numpy(), bits)
        held = R.decode(codes, scales, bits)
        for name, got in (("K", K), ("V", V)):
            assert np.array_equal(h.at(getattr(h.cache, name), 0, 0, np.arange(n)), codes)
            assert np.array_equal(h.at(getattr(h.cache, name + "_scale"), 0, 0, np.arange(n)), scales)
            assert np.array_equal(got[0].double().cpu().numpy(), held, equal_nan=True)
        assert np.array_equal(h.cache.bounds[0, :-(-n // 16)].double().cpu().numpy(), R.bounds_of(held, 16), equal_nan=True)
