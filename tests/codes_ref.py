"""Plain 64-bit forms of the operators over a cache of 8-bit codes and of the scores, on the CPU."""
from __future__ import annotations

import math

import numpy as np
import torch

LOWEST = -40                                             # exponent of a scale


def to_code(x):
    """The nearest value that a code holds (4 significant bits, exponents from 2^-6), ties to even; NaN for what is not finite."""
    x = x.double()
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.where(torch.isfinite(x), torch.round(x / step) * step, torch.nan)


def exponent(most):
    """The smallest whole E >= LOWEST with most <= 448 * 2^E, of 64-bit numbers."""
    part, power = torch.frexp(most)
    return torch.where(most > 0, (power - 9 + (part > 0.875)).clamp(min=LOWEST), LOWEST)


def values(codes, scale):
    """What pools [pages, page, heads, d] stand for, in 64 bits."""
    return codes.cpu().double() * scale.cpu().view(torch.uint8).double().sub(127).exp2()[:, None, :, None]


def pools(seed, n_pages, page, nkv, d, shift=0):
    """Random pages in use, on the CPU: (codes, scales)."""
    g = torch.Generator().manual_seed(seed)
    codes = (torch.randn(n_pages, page, nkv, d, generator=g) * 80).clamp(-448, 448).to(torch.float8_e4m3fn)
    scale = (121 + shift - torch.randint(0, 3, (n_pages, nkv), generator=g)).to(torch.uint8).view(torch.float8_e8m0fnu)
    return codes, scale


def runs(slots, page):
    """The rows of each page, rows without a slot left out."""
    out = []
    for r, x in enumerate(int(x) for x in slots):
        if x >= 0:
            if out and x % page and slots[out[-1][-1]] == x - 1:
                out[-1].append(r)
            else:
                out.append([r])
    return out


def check_append(page, slots, x, size, codes0, scale0, codes, scale):
    """Pools (codes, scale) behind an append of exact values x [rows, heads, d] to (codes0, scale0).  `size`: how far the values that were
    rounded may be off x.  A code is the nearest of a value that is so far off: half a step and that.  The scale is that of
    a largest value that is so far off.  Everything else is what it was, bit for bit."""
    bits, bits0, nkv, d = codes.cpu().view(torch.uint8), codes0.cpu().view(torch.uint8), codes.shape[2], codes.shape[3]
    byte, byte0 = scale.cpu().view(torch.uint8).long(), scale0.cpu().view(torch.uint8).long()
    want, want_byte = bits0.clone(), byte0.clone()
    touched = torch.zeros(bits.shape[:2], dtype=torch.bool)
    for rows in runs(slots, page):
        r, n = rows[0], len(rows)
        p, off = int(slots[r]) // page, int(slots[r]) % page
        y, e = x[rows], size[rows]
        fine = torch.isfinite(y)
        least = torch.where(fine, (y.abs() - e).clamp(min=0), 0.0).amax((0, 2))
        most = torch.where(fine, y.abs() + e, 0.0).amax((0, 2))
        lo, hi = exponent(least) + 127, exponent(most) + 127
        if off:
            lo, hi = torch.maximum(lo, byte0[p]), torch.maximum(hi, byte0[p])
        assert bool(((byte[p] >= lo) & (byte[p] <= hi)).all()), (r, byte[p], lo, hi)
        want_byte[p] = byte[p]
        unit = torch.exp2((byte[p] - 127).double())[None, :, None]
        front = to_code(codes0[p, :off].cpu().double() * torch.exp2((byte0[p] - byte[p]).double())[None, :, None])
        want[p, :off] = front.float().to(torch.float8_e4m3fn).view(torch.uint8)
        got = codes.cpu()[p, off:off + n].double()
        assert bool((torch.isnan(got) == ~fine).all())
        z = torch.where(fine, y / unit, 0.0)
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
        err = torch.where(fine, (got - z).abs() - e / unit, 0.0)
        assert bool((err <= step / 2).all()), f"worst {float((err / step).max()):.4f} of a step"
        exact = torch.where(fine & (e == 0), to_code(z), got)
        assert bool((torch.nan_to_num(got) == torch.nan_to_num(exact)).all())
        touched[p, off:off + n] = True
    assert torch.equal(byte, want_byte)
    assert torch.equal(torch.where(touched[:, :, None, None], 0, bits), torch.where(touched[:, :, None, None], 0, want))


# ---- scores -----------------------------------------------------------------------------------------------------------------
def score(x, token, top):
    """(log-probability, entropy, ids, log-probabilities) of one row of logits, in 64 bits."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    live = np.nonzero(x > -np.inf if x.max() < np.inf else x == np.inf)[0]
    lp = np.full(x.size, -np.inf)
    if live.size:
        z = np.zeros(live.size) if x.max() == np.inf else x[live] - x.max()
        lp[live] = z - math.log(math.fsum(np.exp(z)))
    p = np.exp(lp)
    entropy = -math.fsum(np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0))
    order = np.lexsort((np.arange(x.size), -x))
    order = order[x[order] > -np.inf][:top]
    pad = top - order.size
    return (None if token is None else lp[token], entropy, np.concatenate((order, np.full(pad, -1))).astype(np.int64), np.concatenate((lp[order], np.full(pad, -np.inf))))
