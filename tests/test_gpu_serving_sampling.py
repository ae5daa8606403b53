"""Sampling on the GPU where the filters end: at the largest logit itself, among ties, far behind the tokens that have weight.  Every row
is compared; the inputs keep clear of borders, which is asserted on the 64-bit form."""
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from serving_ref import i32, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def etc():
    import paper_2604_13327_amd
    return paper_2604_13327_amd


def _row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability, kept, gap) of finite logits.  Weights of exactly 1 are in no doubt at min_p: the kernel compares the
    logit with the largest.  The gap is relative to the sums, in which weights are off by 2^-34 of themselves and half of 2^-35."""
    order = np.lexsort((np.arange(x.size), -x))
    w = np.exp((x[order] - x.max()) / temperature)
    n, gap = (min(x.size, top_k) if top_k > 0 else x.size), 1.0
    if top_p < 1:
        c = np.cumsum(w[:n]) / w[:n].sum()
        gap = min(gap, float(np.abs(c - top_p).min()))
        n = min(n, int((c < top_p).sum()) + 1)
    if min_p > 0:
        rest = w[w < 1.0]
        gap = min(gap, float(np.abs(rest - min_p).min()) if rest.size else 1.0)
        n = min(n, max(1, int((w >= min_p).sum())))
    c = np.cumsum(w[:n]) / w[:n].sum()
    if n > 1:
        gap = min(gap, float(np.abs(c[:-1] - u).min()))
    at = min(int((c <= u).sum()), n - 1)
    return int(order[at]), float((x[order[at]] - x.max()) / temperature - math.log(w[:n].sum())), n, gap


def _check(etc, x, u, **settings):
    rows, vocab = x.shape
    u = np.asarray(u, np.float32)
    settings = {k: np.broadcast_to(np.asarray(v, np.int32 if k == "top_k" else np.float32), (rows,)).copy() for k, v in settings.items()}
    want = [_row(x[r].double().numpy(), float(u[r]), **{k: (int if k == "top_k" else float)(v[r]) for k, v in settings.items()}) for r in range(rows)]
    assert min(w[3] for w in want) > 1e-7, "the inputs stand next to a border"
    sv = etc.Serving(ref.shape(vocab=vocab), max_seqs=rows, max_tokens=1, max_kv_len=1)
    token, kept, logprob = i32([-9] * rows), i32([-9] * rows), torch.zeros(rows, device="cuda")
    sv.sample(x.cuda(), torch.as_tensor(u).cuda(), token, logprob_out=logprob, kept_out=kept, **{k: torch.as_tensor(v).cuda() for k, v in settings.items()})
    torch.cuda.synchronize()
    sv.close()
    assert token.tolist() == [w[0] for w in want] and kept.tolist() == [w[2] for w in want]
    # fp32 rounding of the result; the sum of weights is at least 1, each of them off by half of 2^-35 and 2^-34 of itself at most
    for got, (_, p, _, _) in zip(logprob.tolist(), want):
        assert abs(got - p) <= 2.0 ** -24 * abs(p) + 2.0 ** -36 * vocab + 2.0 ** -34


def _clear(make, **settings):
    """Logits and random numbers of the first seed whose rows all keep clear of borders."""
    for seed in range(100):
        x, u = make(seed)
        at = lambda v, r: np.asarray(v).flat[r % np.asarray(v).size]        # noqa: E731
        if all(_row(x[r].double().numpy(), float(np.float32(u[r])), **{k: int(at(v, r)) if k == "top_k" else float(np.float32(at(v, r)))
                                                                      for k, v in settings.items()})[3] > 1e-7 for r in range(x.shape[0])):
            return x, u
    raise AssertionError("no such inputs")


def _u(seed, rows):
    return np.random.default_rng(seed).random(rows, np.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [3, 64, 1000, 16384, 50001])
def test_min_p_of_one_keeps_the_largest_and_its_ties(etc, dtype, vocab):
    rows = 6
    def make(seed):
        x = (randn(seed, rows, vocab, dtype=torch.float32) * 2.5).to(dtype)
        for r, ties in enumerate((1, 2, 3, 40, 70, 9000)):             # as many as fit
            at = np.random.default_rng(seed + r).permutation(vocab)[:ties]
            x[r, torch.as_tensor(at)] = x[r].float().max().to(dtype)
        return x, _u(seed, rows)
    for extra in ({}, {"temperature": 0.25}, {"top_k": 2}, {"top_p": 0.30017}):
        kw = {"min_p": 1.0, **extra}
        x, u = _clear(make, **kw)
        _check(etc, x, u, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1024, 16383, 20000, 128256])
@pytest.mark.parametrize("temperature", [0.02, 0.1, 0.2, 0.3])
def test_top_k_that_ends_behind_all_weight(etc, dtype, vocab, temperature):
    """Low temperatures: the k-th token lies further from the largest than any that has weight."""
    rows, top_k = 4, [20, 50, 1000, 700]
    def make(seed):
        x = randn(seed, rows, vocab, dtype=torch.float32) * 2.5
        x.scatter_add_(1, torch.as_tensor(np.random.default_rng(seed).integers(0, vocab, (rows, 24))), 6.0 + 2.0 * randn(seed + 1, rows, 24, dtype=torch.float32))
        return x.to(dtype), _u(seed, rows)
    for extra in ({}, {"top_p": 0.95}, {"min_p": 0.05}):
        kw = {"temperature": temperature, "top_k": top_k, **extra}
        x, u = _clear(make, **kw)
        _check(etc, x, u, **kw)


def test_rows_of_the_largest_vocabulary(etc):
    vocab = 1 << 20
    make = lambda seed: ((randn(seed, 2, vocab, dtype=torch.float32) * 2.0).bfloat16(), _u(seed, 2))        # noqa: E731
    for kw in ({}, {"temperature": 0.2, "top_k": [40, 5000]}, {"top_p": [0.9, 0.2], "temperature": 0.7}, {"min_p": [0.1, 0.02]}):
        x, u = _clear(make, **kw)
        _check(etc, x, u, **kw)
