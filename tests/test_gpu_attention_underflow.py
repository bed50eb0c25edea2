"""Values that are not finite at keys whose weight is too small for 32 bits.  Whether a query sees a key goes by the
masks: a seen NaN gives NaN also with a weight of 0, and so does a seen infinity (0 times it has no value), in
every form and whatever else is in the tile."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attention import DEV, _batch, _randn, check_decode, check_prompt

pytestmark = pytest.mark.gpu

FORMS = [([300], [300], 4, 2), ([300], [9], 4, 2), ([700, 700, 701], [700, 700, 690], 12, 6),
         ([400, 1, 0, 399, 400, 380], [200, 1, 0, 200, 200, 199], 32, 8), ([3999], [301], 16, 2),
         ([400, 390, 400, 400, 370, 400], [200, 190, 200, 200, 170, 200], 32, 8), ([6000], [3000], 4, 2)]


@pytest.mark.parametrize("docs", [0, 150])
@pytest.mark.parametrize("lens,new,hq,hkv", FORMS)
def test_seen_nan_without_a_weight(lens, new, hq, hkv, docs):
    """Scores of hundreds: most weights are 0, and a NaN value still reaches the queries that see it and no others."""
    def spoil(K, V):
        K.mul_(64.0)
        n, m = lens[0], new[0]
        V[0, n - m // 2, 5] = float("nan")
        V[1, max(n - m // 2 - 70, 0):n - m // 2 - 5:9, 17] = float("nan")
    check_prompt(lens, new, hq, hkv, docs=docs, spoil=spoil)


@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("odd", [False, True])
def test_seen_infinity_without_a_weight(value, odd):
    """Key 10 has a score 600 under the others': its infinite value gives NaN to all that see it, whether the item
    holds masked values that are not finite as well (odd) or not."""
    import paper_2502_12216_amd as T
    n, hq, hkv = 400, 4, 2
    batch = _batch([n], hq, hkv)
    K, V, q = torch.zeros(hkv, n, 128, dtype=torch.bfloat16, device=DEV), _randn(2, hkv, n, 128), torch.ones(n, hq, 128, dtype=torch.bfloat16, device=DEV)
    K[:, 10] = -53.0  # a score of -53 sqrt(128) = -599.6
    clean = V.clone()
    V[:, 10, 3] = value
    if odd:
        V[:, 390, 7] = float("nan")
    out, _ = T.PromptAttention(batch, [n])(q, K, V)
    torch.cuda.synchronize()
    ref, _ = T.PromptAttention(batch, [n])(q, K, clean)
    want = torch.zeros(n, 128, dtype=torch.bool, device=DEV)
    want[11:, 3] = True  # (query 10 sees 11 keys, ten of which have all the weight; queries before it do not see it)
    want[10, 3] = True
    if odd:
        want[390:, 7] = True
    for h in range(hq):
        assert torch.equal(torch.isnan(out[:, h]), want), h
        assert torch.equal(out[:, h][~want], ref[:, h][~want]), h
    pos, seen = torch.arange(n, device=DEV), torch.arange(n, device=DEV)[None] <= torch.arange(n, device=DEV)[:, None]
    for h in range(hq):
        o, _, _, ma, off = R.attend(q[:, h], K[h // 2], clean[h // 2], pos, pos, seen)
        R.close(ref[:, h], o, R.tolerance_bf16(ma, off, o), f"h={h}")


@pytest.mark.parametrize("kw", [dict(), dict(docs=90), dict(alibi=True, positions=True, add=True), dict(page=16, cap=500.0), dict(page=7, docs=300)])
@pytest.mark.parametrize("lens", [[700, 1, 0, 2049], [33000]])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
def test_decode_of_seen_nan_without_a_weight(hq, hkv, lens, kw):
    """Scores of hundreds: a NaN value reaches the query that sees it from any lane group, wave or split."""
    def spoil(K, V, document, qd):
        K.mul_(64.0)
        V[0, 3, 5], V[0, 500, 6], V[0, 640:699, 8] = (float("nan"),) * 3
        V[1, 650, 64] = float("nan")
    check_decode(lens, hq, hkv, spoil=spoil, **kw)


def test_decode_of_seen_nan_where_the_last_rows_have_all_the_weight():
    """A share of the rows, and every lane group of it but the last, has a weight of 0."""
    def spoil(K, V, document, qd):
        K[:, :-1] *= 200.0
        V[:, 10::1000, 3] = float("nan")
    check_decode([33000], 8, 2, spoil=spoil)
