"""Attention with capped and biased scores, masks, sums and evictions in 64 bits,
and the error that 32-bit sums of bf16 products may have (test infrastructure)."""
import numpy as np
import torch

D = 128


def slopes(hq, device="cuda"):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=device)


def attend(q, k, v, qpos, kpos, seen, cap=0.0, slope=0.0):
    """One query head: q [m][128], k, v [n][128] bf16; qpos [m], kpos [n]; seen bool [m][n].

    Returns out [m][128], lse [m], weights [m][n] and per row: |v| averaged by the weights [m][128], and the
    bound `off` on how far a computed logit may be: 130 roundings of the 128 products' absolute sum (fp32
    accumulation in any order), 8 roundings each of the score, the cap's value and the bias (transforms and the
    argument of the exponential, which has a magnitude of at most |score - lse|)."""
    q, k = q.double(), k.double()
    v = torch.where(seen.any(0)[:, None], v.double(), 0.0)  # a value that no row sees has no weight, also as NaN
    k = torch.where(seen.any(0)[:, None], k, 0.0)
    s = q @ k.T / D ** 0.5
    absolute = torch.where(seen, q.abs() @ k.abs().T / D ** 0.5, 0.0)
    u = 2.0 ** -24
    off = 130 * u * absolute
    if cap:
        s = cap * torch.tanh(s / cap)
        off = off + 8 * u * s.abs()
    dist = (qpos[:, None] - kpos[None, :]).abs().double()
    s = s - slope * dist
    off = off + 8 * u * (s.abs() + slope * dist)
    s = torch.where(seen, s, -np.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - lse[:, None]), 0.0)
    off = torch.where(seen, off + 8 * u * (s - torch.where(lse == -np.inf, 0.0, lse)[:, None]).abs(), 0.0)
    # rows may see different keys: those of a row's own
    out = torch.stack([p[i] @ torch.where(seen[i][:, None], v, 0.0) for i in range(len(p))]) if torch.isnan(v).any() or \
        torch.isinf(v).any() else p @ v
    mean_abs = p @ torch.nan_to_num(v, 0.0, 0.0, 0.0).abs()
    return out, lse, p, mean_abs, off.amax(1) if off.shape[1] else torch.zeros(len(q), dtype=torch.float64, device=q.device)


def tolerance_fp32(mean_abs, off, out):
    """A weight's relative error is at most e^{2 off} - 1 (its own logit and the sum's); sums and the quotient: 64
    roundings of the absolute sum (accumulation over tiles, waves and splits, each of few terms in order)."""
    u = 2.0 ** -24
    return mean_abs * (2.1 * off[:, None] + 64 * u) + 4 * u * out.abs() + 1e-30


def tolerance_bf16(mean_abs, off, out):
    """As above, with the weights rounded to bf16 (2^-8 of each) and the output once (2^-8)."""
    return tolerance_fp32(mean_abs, off, out) + 2.0 ** -8 * (1 + 2.0 ** -8) * (mean_abs + out.abs())


def tolerance_lse(off, lse):
    return off + 2.0 ** -24 * (64 + 8 * torch.where(lse == -np.inf, 0.0, lse).abs())


def close(got, ref, tol, what):
    got = got.double()
    assert got.shape == ref.shape, what
    odd = ~torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN elsewhere"
    assert torch.equal(got[odd & ~torch.isnan(ref)], ref[odd & ~torch.isnan(ref)]), f"{what}: infinities elsewhere"
    err = torch.where(odd, 0.0, (got - torch.where(odd, 0.0, ref)).abs())
    bad = err > torch.broadcast_to(tol, err.shape)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((err / tol).max()):.2f} of it"
    return float((err / tol.clamp_min(1e-30)).max()) if err.numel() else 0.0


def ranking(weights, positions, newest, recent):
    """Rows of one KV head from the first to keep to the last (numpy): recent by position, then weight (NaN last), ties by row."""
    n = len(weights)
    age = np.int64(newest) - positions.astype(np.int64)
    fresh = age < recent
    w = np.where(np.isnan(weights), -np.inf, weights.astype(np.float64))
    return np.lexsort((np.arange(n), np.isnan(weights) & ~fresh, np.where(fresh, 0.0, -w), np.where(fresh, age, 2 ** 40)))


def pages(x, lens, page, order_seed=0):
    """Pages [pages][hkv][page][128] of x [hkv][total][128] in shuffled places, and the table [B][max]."""
    counts = [max(1, -(-n // page)) for n in lens]
    place = torch.as_tensor(np.random.default_rng(order_seed).permutation(sum(counts)).astype(np.int32), device=x.device)
    table = torch.zeros(len(lens), max(counts), dtype=torch.int32, device=x.device)
    out = torch.full((sum(counts), x.shape[0], page, D), float("nan"), dtype=x.dtype, device=x.device)
    at = 0
    for b, ids in enumerate(place.split(counts)):
        table[b, :len(ids)] = ids
        for i, p in enumerate(ids.tolist()):
            rows = x[:, at + i * page:at + min((i + 1) * page, lens[b])]
            out[p, :, :rows.shape[1]] = rows
        at += lens[b]
    return out, table
