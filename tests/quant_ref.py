"""The quantised cache, blocks chosen by their bounds, and attention over both, plainly and in 64 bits
(test infrastructure)."""
import numpy as np
import torch

from attention_ref import attend

D = 128
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3(code):
    """Values of e4m3 codes (numpy)."""
    code = np.asarray(code).astype(np.int64)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(code >> 7, -v, v)


def numbers(bits):
    """The numbers >= 0 of a format in the order of their codes."""
    return e4m3(np.arange(127)) if bits == 8 else E2M1


def encode(x, bits):
    """Codes uint8 [n][16 bits] and scales uint8 [n][4] of x float64 [n][128] (bf16 values, numpy)."""
    table = numbers(bits)
    least, most = (-117, 119) if bits == 8 else (-125, 125)
    codes = np.zeros(x.shape, np.uint8)
    scales = np.zeros((len(x), 4), np.uint8)
    for c in range(4):
        g = x[:, 32 * c:32 * c + 32]
        bad = ~np.isfinite(g).all(1)
        amax = np.where(bad, 0.0, np.abs(np.where(np.isfinite(g), g, 0.0)).max(1))
        s = np.full(len(x), least)
        for p in range(least, most):  # the least power that holds it
            s = np.where(amax > table[-1] * 2.0 ** p, p + 1, s)
        y = np.where(bad[:, None], 0.0, np.where(np.isfinite(g), g, 0.0) * 2.0 ** -s[:, None].astype(float))
        a = np.minimum(np.abs(y), table[-1])
        hi = np.searchsorted(table, a).clip(0, len(table) - 1)  # the first number >= a
        lo = np.maximum(hi - 1, 0)
        up, down = table[hi] - a, a - table[lo]
        code = np.where(up < down, hi, np.where(down < up, lo, np.where(lo % 2 == 0, lo, hi)))
        code = np.where(table[hi] == a, hi, code)
        neg = np.signbit(y)
        codes[:, 32 * c:32 * c + 32] = code | (neg.astype(np.int64) << (7 if bits == 8 else 3))
        scales[:, c] = np.where(bad, 255, s + 127)
    if bits == 4:
        codes = codes[:, ::2] | (codes[:, 1::2] << 4)
    return codes, scales


def decode(codes, scales, bits):
    """Values float64 [..][128] of codes and scales (numpy)."""
    if bits == 8:
        v = e4m3(codes)
    else:
        c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], D)
        v = np.where(c & 8, -E2M1[c & 7], E2M1[c & 7])
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(float) - 127))
    return v * np.repeat(power, 32, axis=-1)


def bounds_of(values, block):
    """[blocks][2][128] of the rows values [n][128] of one sequence; NaN where a row has one."""
    out = []
    for i in range(0, len(values), block):
        part = values[i:i + block]
        out.append(np.stack([part.min(0), part.max(0)]))
    return np.array(out).reshape(-1, 2, D)


def choose(q, bounds, budget, first, last):
    """Blocks (ascending) for q [G][128] from bounds [nb][2][128], float64 (numpy)."""
    nb = len(bounds)
    score = np.full(nb, -np.inf)
    odd = np.zeros(nb, bool)
    with np.errstate(invalid="ignore"):
        for row in q:
            u = np.where(row < 0, row * bounds[:, 0], row * bounds[:, 1]).sum(1)
            d = u - (np.nanmax(u) if not np.isnan(u).all() else -np.inf)
            odd |= np.isnan(d)
            score = np.fmax(score, d)
    score[odd] = np.inf
    i = np.arange(nb)
    always = (i < first) | (i >= nb - last)
    return np.sort(np.lexsort((i, -score, ~always))[:budget])


def rows_of_blocks(chosen, block, n):
    return np.concatenate([np.arange(j * block, min(n, j * block + block)) for j in chosen] or [np.zeros(0, np.int64)])


def one_token(q, k, v, rows, n, cap=0.0, slope=0.0):
    """attend() of one query over rows of a sequence of n; k, v float64 tensors [rows][128]."""
    seen = torch.ones(1, len(rows), dtype=torch.bool, device=q.device)
    return attend(q[None], k, v, torch.tensor([n - 1], device=q.device), torch.as_tensor(rows, device=q.device), seen, cap, slope)


def tolerance(mean_abs, off, out, rows):
    """A weight's relative error is at most e^{2 off} - 1.  Sums: a weight's three parts are added one after another, 32
    rows to a step of a wave (up to rows / 32 steps), and 64 states, splits and quotients follow."""
    u = 2.0 ** -24
    return mean_abs * (2.1 * off[:, None] + (3 * (rows / 32 + 1) + 64) * u) + 4 * u * out.abs() + 1e-30


def tolerance_lse(off, lse, rows):
    return off + 2.0 ** -24 * (rows / 32 + 64 + 8 * torch.where(lse == -np.inf, 0.0, lse).abs())
