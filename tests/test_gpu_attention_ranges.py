"""Scores over the whole range of their parameters: caps far from the usual ones, against the plain 64-bit
implementation (tests/attention_ref.py) or, where a cap is so small that every weight is the same, its formula."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attention import DEV, _batch, _randn, check_decode, check_prompt

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _weights(att, q, K, V, mod, lse):
    """Sums of every query's weights against 64 bits, with the lse that the call was given (one sequence)."""
    n, hq, hkv = q.shape[0], q.shape[1], K.shape[0]
    got = att.add_weights(q, K, lse, torch.zeros(hkv, n, device=DEV), mod)
    torch.cuda.synchronize()
    pos = torch.arange(n, device=DEV)
    seen = pos[None] <= pos[:, None]
    ref, slack = (torch.zeros(hkv, n, dtype=torch.float64, device=DEV) for _ in range(2))
    for h in range(hq):
        g = h * hkv // hq
        _, l, p, _, off = R.attend(q[:, h], K[g], V[g], pos, pos, seen, mod.cap)
        p = p * torch.exp(l - lse[h].double())[:, None]
        ref[g] += p.sum(0)
        # the logit, and the roundings of the base-2 score, the logarithm and their difference
        slack[g] += (p * (1.1 * off + U * (16 + 8 * l.abs()))[:, None]).sum(0)
    # (a weight below the least normal number of 32 bits, 2^-126, may be missing)
    R.close(got, ref, slack + (n * hq / hkv / 16 + 64) * U * ref + n * hq / hkv * 2.0 ** -126, "sums")


@pytest.mark.parametrize("cap", [60.0, 300.0, 700.0, 2e4, 1e5, 1e9])
def test_caps_larger_than_the_usual(cap):
    """Scores up to about 0.7 of the cap, where its polynomial's highest terms count."""
    def spoil(K, V):
        K.mul_(cap / 10)
    att, q, K, V, mod, out, lse, _ = check_prompt([500], [500], 4, 2, cap=cap, spoil=spoil)
    if cap < 1e6:  # (a logarithm of 2^29 has a rounding of 2^4 in 32 bits: no weight follows from it)
        _weights(att, q, K, V, mod, lse)
    check_decode([500], 4, 2, cap=cap, spoil=lambda K, V, d, q: spoil(K, V))


@pytest.mark.parametrize("cap", [300.0, 2e4, 1e9])
def test_caps_of_a_shared_prefix_larger_than_the_usual(cap):
    import paper_2502_12216_amd as T
    hq, hkv, n = 8, 2, 400
    batch = _batch([0, 0], hq, hkv)
    own = torch.zeros(hkv, 0, 128, dtype=torch.bfloat16, device=DEV)
    K, V, q = _randn(1, hkv, n, 128, scale=cap / 10), _randn(2, hkv, n, 128), _randn(3, 2, hq, 128, scale=2.0)
    out, lse = T.SharedPrefixDecoder(batch, [n], [0, 0])(q, K, V, own, own, T.ScoreMod(cap=cap))
    torch.cuda.synchronize()
    pos, seen = torch.arange(n, device=DEV), torch.ones(2, n, dtype=torch.bool, device=DEV)
    for h in range(hq):
        o, l, _, ma, off = R.attend(q[:, h], K[h // 4], V[h // 4], pos[-1:].expand(2), pos, seen, cap)
        R.close(out[:, h], o, R.tolerance_fp32(ma, off, o), f"out h={h}")
        R.close(lse[:, h], l, R.tolerance_lse(off, l), f"lse h={h}")


@pytest.mark.parametrize("cap", [2.0 ** -120, 1e-12, 1e-8, 1e-6])
def test_caps_so_small_that_every_weight_is_the_same(cap):
    """Scores lie within the cap, so that the weights differ by less than 2 cap; the scores of whole tiles are exactly 0."""
    import paper_2502_12216_amd as T
    n, hq, hkv = 300, 4, 2
    batch = _batch([n], hq, hkv)
    K, V, q = _randn(1, hkv, n, 128), _randn(2, hkv, n, 128), _randn(3, n, hq, 128)
    K[:, :200] = 0.0  # (whole tiles whose scores are 0)
    mod = T.ScoreMod(cap=cap)
    att = T.PromptAttention(batch, [n])
    out, lse = att(q, K, V, mod)
    sums = att.add_weights(q, K, lse, torch.zeros(hkv, n, device=DEV), mod)
    o1, l1 = T.ScoredDecoder(batch)(q[-1:].contiguous(), K, V, mod)
    pre = T.SharedPrefixDecoder(_batch([0], hq, hkv), [n], [0])
    own = torch.zeros(hkv, 0, 128, dtype=torch.bfloat16, device=DEV)
    o2, l2 = pre(q[-1:].contiguous(), K, V, own, own, mod)
    torch.cuda.synchronize()
    seen = torch.arange(1, n + 1, dtype=torch.float64, device=DEV)
    for h in range(hq):
        v = V[h // 2].double()
        mean, size = (x.cumsum(0) / seen[:, None] for x in (v, v.abs()))
        tol = size * (2.1 * cap + 64 * U) + 1e-30
        R.close(out[:, h], mean, tol + 2.0 ** -8 * (1 + 2.0 ** -8) * (size + mean.abs()), f"out h={h}")
        R.close(lse[h], seen.log(), cap + U * (64 + 8 * seen.log()), f"lse h={h}")
        for o, l in ((o1, l1), (o2, l2)):
            R.close(o[0, h], mean[-1], tol[-1], f"decode h={h}")
            R.close(l[0, h:h + 1], seen[-1:].log(), cap + U * (64 + 8 * seen[-1:].log()), f"decode lse h={h}")
    want = 2 * (1 / seen).flip(0).cumsum(0).flip(0)  # two heads per KV head
    R.close(sums, want.expand(hkv, n), want * (2.1 * cap + U * (16 + 8 * 6 + n * 2 / 16 + 64)), "sums")


@pytest.mark.parametrize("cap", [2.0 ** 120, 1e30, 1e20])
def test_caps_beyond_every_score(cap):
    check_prompt([300], [300], 4, 2, cap=cap)
    check_decode([300], 4, 2, cap=cap)
    check_prompt([300], [300], 4, 2, cap=cap, spoil=lambda K, V: K.mul_(1e18))


@pytest.mark.parametrize("window", [0, 260])
@pytest.mark.parametrize("kw", [dict(), dict(docs=70), dict(cap=20.0, alibi=True)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_weights_of_queries_that_give_none(value, kw, window):
    """A logarithm of -inf takes a query out whatever the query holds: padding, or heads that a caller leaves out."""
    import paper_2502_12216_amd as T
    n, hq, hkv = 300, 8, 2
    batch = _batch([n], hq, hkv)
    K, V, q = _randn(1, hkv, n, 128), _randn(2, hkv, n, 128), _randn(3, n, hq, 128)
    document = torch.arange(n, dtype=torch.int32, device=DEV) // kw["docs"] if "docs" in kw else None
    mod = T.ScoreMod(cap=kw.get("cap", 0.0), documents=document, slopes=R.slopes(hq) if "alibi" in kw else None)
    att = T.PromptAttention(batch, [n])
    _, lse = att(q, K, V, mod)
    lse = lse.clone()
    out = torch.zeros(hq, n, dtype=torch.bool, device=DEV)
    out[1, 50], out[6, 210], out[:, 297:], out[3, 64:192] = True, True, True, True
    lse[out] = -float("inf")
    want = att.add_weights(q, K, lse, torch.zeros(hkv, n, device=DEV), mod, window=window).clone()
    q[out.T] = value
    got = att.add_weights(q, K, lse, torch.zeros(hkv, n, device=DEV), mod, window=window)
    torch.cuda.synchronize()
    assert torch.isfinite(want).all() and torch.equal(got, want)
    assert not want[:, 297:].any()


@pytest.mark.parametrize("positions", [True, False])
@pytest.mark.parametrize("qp", [2 ** 31 - 1, 0, -2 ** 31])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (16, 2)])
def test_distances_that_pass_31_bits(hq, hkv, qp, positions):
    """Positions over the whole range of int32: the bias goes by their true distance."""
    import paper_2502_12216_amd as T
    n = 200
    batch = _batch([n], hq, hkv)
    K, V, q = _randn(1, hkv, n, 128), _randn(2, hkv, n, 128), _randn(3, 1, hq, 128)
    slopes = torch.linspace(1.0, 2.0, hq, device=DEV) * 2.0 ** -30
    pos = torch.linspace(-2.0 ** 31, 2.0 ** 31 - 1, n, dtype=torch.float64, device=DEV).round().to(torch.int64)
    pos = torch.stack([pos, pos.flip(0)])
    kw = dict(positions=pos.to(torch.int32).contiguous()) if positions else {}
    out, lse = T.ScoredDecoder(batch)(q, K, V, T.ScoreMod(slopes=slopes), q_pos=torch.tensor([qp], dtype=torch.int32, device=DEV), **kw)
    torch.cuda.synchronize()
    for h in range(hq):
        g = h * hkv // hq
        kpos = pos[g] if positions else torch.arange(n, device=DEV)
        o, l, _, ma, off = R.attend(q[:, h], K[g], V[g], torch.tensor([qp], device=DEV), kpos, torch.ones(1, n, dtype=torch.bool, device=DEV),
                                    0.0, float(slopes[h]))
        R.close(out[:, h], o, R.tolerance_fp32(ma, off, o), f"out h={h}")
        R.close(lse[:, h], l, R.tolerance_lse(off, l), f"lse h={h}")
