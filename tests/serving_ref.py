"""Plain 64-bit forms of the serving operators, on the CPU, and what their tests share."""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch


def shape(nq=4, nkv=2, d=64, page=16, qk_norm=False, vocab=0, theta=1e4, eps=1e-5):
    return SimpleNamespace(n_layers=1, H=nq * d, nq=nq, nkv=nkv, d=d, F=0, n_experts=0, top_k=0, moe_F=0, page=page, eps=eps,
                           theta=theta, qk_norm=qk_norm, vocab=vocab)


def pages_needed(n, page):
    return -(-int(n) // page)


def i32(x, device="cuda"):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).to(device)


def randn(seed, *size, dtype=torch.bfloat16):
    return torch.randn(*size, generator=torch.Generator().manual_seed(seed)).to(dtype)


# ---- page tables --------------------------------------------------------------------------------------------------------
def tables(kv, new, table, free, page, n_rows):
    """What etc_serving_tables leaves, as a dict of numpy arrays; `free` a list that is consumed from its end."""
    table, free = np.array(table), list(free)
    q, pi, slots, pos, ids = [0], [0], [], [], []
    for b, (k, n) in enumerate(zip(kv, new)):
        for p in range(pages_needed(k, page), pages_needed(k + n, page)):
            table[b, p] = free.pop()
        for t in range(k, k + n):
            slots.append(int(table[b, t // page]) * page + t % page)
            pos.append(t)
        ids += list(table[b, :pages_needed(k + n, page)])
        q.append(len(slots))
        pi.append(len(ids))
    pad = n_rows - len(slots)
    return {"block_table": table, "free_count": [len(free)], "q_indptr": q, "slots": slots + [-1] * pad, "positions": pos + [0] * pad,
            "total_len": [k + n for k, n in zip(kv, new)], "page_indptr": pi, "page_ids": ids, "status": [0]}


def paged(kv_and_new, page, seed, extra=3):
    """A random page table with room for the given totals: (table, number of pages)."""
    rng = np.random.default_rng(seed)
    need = [pages_needed(n, page) for n in kv_and_new]
    n_pages = sum(need) + extra
    ids = rng.permutation(n_pages)
    table = np.zeros((len(need), max(need + [1]) + 1), np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, n_pages


# ---- append ---------------------------------------------------------------------------------------------------------------
def rotate(s, x, positions, gain=None):
    """Norm and rotation of heads x [tokens, heads, d] in 64 bits; also the size of what a rotated element is the sum of."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + s.eps) * gain.double()
    ang = torch.as_tensor(positions).double()[:, None] * s.theta ** (-2.0 * torch.arange(s.d // 2).double() / s.d)
    c, sn = ang.cos()[:, None], ang.sin()[:, None]
    a, b = x[..., :s.d // 2], x[..., s.d // 2:]
    return torch.cat((a * c - b * sn, a * sn + b * c), -1), (a.abs() + b.abs()).repeat(1, 1, 2)


# ---- attention --------------------------------------------------------------------------------------------------------------
def attention(s, q, k_pages, v_pages, q_indptr, kv_len, table):
    """(out, sum of softmax * |v|) in 64 bits, CPU; only what a row sees takes part."""
    k_pages, v_pages = k_pages.cpu(), v_pages.cpu()
    q = q.cpu().double()
    out = torch.zeros(q.shape, dtype=torch.float64)
    size = torch.zeros_like(out)
    g = s.nq // s.nkv
    for b in range(len(kv_len)):
        n, kv = int(q_indptr[b + 1] - q_indptr[b]), int(kv_len[b])
        if n == 0:
            continue
        slot = torch.arange(kv + n)
        page = torch.as_tensor(np.asarray(table[b]).astype(np.int64))[slot // s.page]
        k, v = k_pages[page, slot % s.page].double(), v_pages[page, slot % s.page].double()     # [keys, nkv, d]
        seen = slot[None, :] <= kv + torch.arange(n)[:, None]
        rows = slice(int(q_indptr[b]), int(q_indptr[b + 1]))
        for h in range(s.nq):
            score = torch.where(seen, (q[rows, h] @ k[:, h // g].t()) / math.sqrt(s.d), -math.inf)
            p = score.softmax(-1)
            vv = v[:, h // g]
            if bool(torch.isfinite(vv).all()):
                out[rows, h], size[rows, h] = p @ vv, p @ vv.abs()
            else:                                       # what a row does not see is no part of its sum
                for t in range(n):
                    out[rows.start + t, h] = (p[t, :kv + t + 1, None] * vv[:kv + t + 1]).sum(0)
                    size[rows.start + t, h] = (p[t, :kv + t + 1, None] * vv[:kv + t + 1].abs()).sum(0)
    return out, size


def check_attention(got, out, size):
    """Elementwise: probabilities are rounded to bf16 once (half a step, 2^-8 of each: 2^-8 sum p |v|), the result once (2^-8 of it).
    Scores, exponentials and sums are fp32: a score of up to about 10 in units of log2 from 128 products is off by 128 * 2^-24 of the
    sum of their sizes (about 8 times the score) at most, 2^-14 of the weight, numerator and denominator: below 2^-12 sum p |v|."""
    got = got.double().cpu()
    assert torch.equal(torch.isfinite(got), torch.isfinite(out))
    fin = torch.isfinite(out)
    err = (got - out).abs()[fin]
    bound = (2.0 ** -8 * (out.abs() + size) + 2.0 ** -12 * size)[fin] + 1e-30
    assert bool((err <= bound).all()), f"worst error / bound {float((err / bound).max()):.3f}"


# ---- sampling ---------------------------------------------------------------------------------------------------------------
def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability, kept, gap): gap is how far the draw and the filters are from a border, relative to the sums."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    if x.max() == -np.inf:
        return -1, -math.inf, 0, 1.0
    order = np.lexsort((np.arange(x.size), -x))
    if not temperature > 0:
        return int(order[0]), 0.0, 1, 1.0
    live = int((x == np.inf).sum()) if x.max() == np.inf else int((x > -np.inf).sum())
    z = np.zeros(live) if x.max() == np.inf else (x[order[:live]] - x.max()) / float(temperature)
    w, gap = np.exp(z), 1.0
    n = min(live, int(top_k)) if top_k > 0 else live
    if top_p < 1:
        c = np.cumsum(w[:n])
        gap = min(gap, float(np.abs(c / c[-1] - max(float(top_p), 0.0)).min()))
        n = min(n, int((c < max(float(top_p), 0.0) * c[-1]).sum()) + 1)
    if min_p > 0:
        gap = min(gap, float(np.abs(w - float(min_p)).min()))
        n = min(n, max(1, int((w >= float(min_p)).sum())))
    c = np.cumsum(w[:n]) / w[:n].sum()
    gap = min(gap, float(np.abs(c - u)[:-1].min()) if n > 1 else 1.0)
    at = min(int((c <= u).sum()), n - 1)
    return int(order[at]), float(z[at] - math.log(w[:n].sum())), n, gap
