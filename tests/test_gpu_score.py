"""Log-probabilities of given tokens, entropy and likeliest tokens on the GPU, against their plain 64-bit form on the CPU."""
import math

import numpy as np
import pytest
import torch

import codes_ref as codes
import serving_ref as ref
from serving_ref import i32, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def etc():
    import paper_2604_13327_amd
    return paper_2604_13327_amd


def _run(etc, x, tokens, top, entropy=True, tops=True, max_seqs=None, stride=0, offset=0, serving=None):
    """x [rows, vocab] on the CPU; rows `stride` elements longer in memory, the first one `offset` elements behind an aligned place."""
    rows, vocab = x.shape
    wide = torch.full((rows * (vocab + stride) + offset + 8,), 9.0, dtype=x.dtype, device="cuda")      # larger than most: not to be read
    view = wide[offset:offset + rows * (vocab + stride)].view(rows, vocab + stride)[:, :vocab]
    view.copy_(x)
    sv = serving or etc.Serving(ref.shape(vocab=vocab), max_seqs=min(1024, max_seqs or rows), max_tokens=rows, max_kv_len=1)
    out = {"logprob": torch.full((rows,), 55.0, device="cuda"), "entropy": torch.full((rows,), 55.0, device="cuda"),
           "ids": torch.full((rows, top), 55, dtype=torch.int32, device="cuda"), "tops": torch.full((rows, top), 55.0, device="cuda")}
    sv.score(view, None if tokens is None else i32(tokens), None if tokens is None else out["logprob"], out["entropy"] if entropy else None,
             out["ids"] if top else None, out["tops"] if top and tops else None)
    torch.cuda.synchronize()
    if serving is None:
        assert sv.read_error() == (0, 0, 0, 0)
        sv.close()
    return {k: v.cpu().numpy() for k, v in out.items()}


def _check(x, tokens, top, got, rows=None):
    """A thread adds at most 32 weights and then at most 16 such sums (longer rows than 2^17: 2^(-24) for each 8192 more), all positive: 48
    roundings of 2^-24, and at most 18 more across a wavefront, wavefronts and slices; a weight has an exponent rounded at up to 2^5 (2^-19) and an instruction's unit (2^-23): the sum is within 2^-17,
    and so is its logarithm; the result is rounded once.  The sum of p ln p likewise, relative to the sum of p |ln p|, counted from a
    reference within 6 of the largest."""
    for r in range(x.shape[0]) if rows is None else rows:
        if tokens is not None and tokens[r] < 0:
            assert got["logprob"][r] == 55.0 and got["entropy"][r] == 55.0 and (got["ids"][r] == 55).all() and (got["tops"][r] == 55.0).all()
            continue
        lp, entropy, ids, tops = codes.score(x[r].double().numpy(), None if tokens is None else int(tokens[r]), top)
        close = lambda a, b, tol: a == b or abs(a - b) <= tol      # noqa: E731
        if tokens is not None:
            assert close(got["logprob"][r], lp, 2.0 ** -17 + 2.0 ** -23 * abs(lp)), (r, got["logprob"][r], lp)
        if got["entropy"][r] != 55.0:
            assert close(got["entropy"][r], entropy, 2.0 ** -17 * (8 + entropy)), (r, got["entropy"][r], entropy)
        assert np.array_equal(got["ids"][r], ids), (r, got["ids"][r], ids)
        assert all(close(a, b, 2.0 ** -17 + 2.0 ** -23 * abs(b)) for a, b in zip(got["tops"][r], tops)), (r, got["tops"][r], tops)


def _logits(seed, rows, vocab, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * 2.5
    return x.scatter_add(1, torch.randint(0, vocab, (rows, 8), generator=g), 6 + 2 * torch.randn(rows, 8, generator=g)).to(dtype)


def _tokens(seed, rows, vocab):
    return np.random.default_rng(seed).integers(0, vocab, rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 5), (2, 7, 64), (5, 63, 20), (1, 1000, 5), (4, 1024, 64), (2, 16383, 20), (2, 16384, 20),
                                            (1, 50257, 64), (17, 128256, 20), (300, 1111, 3), (257, 20001, 1), (130, 20001, 7), (2, 1 << 20, 33)])
def test_score(etc, dtype, rows, vocab, top):
    x, tokens = _logits(rows + vocab, rows, vocab, dtype), _tokens(vocab, rows, vocab)
    _check(x, tokens, top, _run(etc, x, tokens, top), rows=range(0, rows, max(1, rows // 20)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,stride,offset", [(1001, 0, 1), (1001, 7, 3), (20003, 1, 5), (5, 3, 1), (9, 0, 7)])
def test_score_alignment(etc, dtype, vocab, stride, offset):
    x, tokens = _logits(vocab, 6, vocab, dtype), _tokens(1, 6, vocab)
    _check(x, tokens, 12, _run(etc, x, tokens, 12, stride=stride, offset=offset))


@pytest.mark.parametrize("vocab", [500, 30000])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_score_shapes_of_rows(etc, vocab, top):
    """Rows that keep a list busy: rising, falling, flat, few different values, all banned but some, far from zero, steep."""
    n = torch.arange(vocab).float()
    g = torch.Generator().manual_seed(vocab)
    few = torch.full((vocab,), -math.inf)
    few[torch.randint(0, vocab, (9,), generator=g)] = 1.5
    end = torch.full((vocab,), -math.inf)
    end[-1] = -3e38
    x = torch.stack((n / vocab, -n / vocab, torch.zeros(vocab), torch.randint(0, 3, (vocab,), generator=g).float(), few, torch.randn(vocab, generator=g) + 1e4,
                     torch.randn(vocab, generator=g) - 3e4, torch.randn(vocab, generator=g) * 1000, n, end, torch.full((vocab,), -0.0) + (n % 2) * 0.0,
                     torch.randn(vocab, generator=g) * 1e-3))
    for y in (x, x.bfloat16()):
        tokens = _tokens(2, y.shape[0], vocab)
        _check(y, tokens, top, _run(etc, y, tokens, top))


@pytest.mark.parametrize("vocab", [300, 40000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_score_no_numbers(etc, vocab, dtype):
    x = _logits(5, 12, vocab, dtype)
    lowest = torch.finfo(dtype).min
    x[0, ::3], x[1, :] = math.nan, -math.inf
    x[2, :] = math.nan
    x[3, 7], x[3, vocab - 1] = math.inf, math.inf
    x[4, 11] = math.inf
    x[5, :] = lowest
    x[6, 1:] = lowest
    x[7, :] = lowest
    x[7, 5] = -torch.finfo(dtype).max / 2
    x[8, 9] = torch.finfo(dtype).max
    x[9, :], x[9, 3] = -math.inf, -2.0
    x[10, :vocab // 2] = -math.inf
    x[11, 5], x[11, 6] = torch.finfo(dtype).max, math.nan
    x.view(torch.int32 if dtype == torch.float32 else torch.int16)[0, 1] = 0x7F800001 if dtype == torch.float32 else 0x7F81      # a signalling NaN
    for tokens in (np.full(12, 7), np.array([0, 1, 2, 3, 11, 5, 0, 5, 9, 3, 0, 6])):
        _check(x, tokens, 9, _run(etc, x, tokens, 9))


def test_score_what_is_asked_for(etc):
    x, tokens = _logits(1, 5, 2000), np.array([3, -1, 5, -7, 1999])
    _check(x, tokens, 6, _run(etc, x, tokens, 6))
    _check(x, tokens, 0, _run(etc, x, tokens, 0))
    _check(x, None, 6, _run(etc, x, None, 6))
    got = _run(etc, x, None, 6, entropy=False, tops=False)
    assert (got["entropy"] == 55.0).all() and (got["tops"] == 55.0).all() and np.array_equal(got["ids"], _run(etc, x, None, 6)["ids"])
    sv = etc.Serving(ref.shape(vocab=2000), max_seqs=1, max_tokens=5, max_kv_len=1)
    tokens[2] = 2000
    got = _run(etc, x, tokens, 6, serving=sv)
    assert sv.read_error() == (4, 7, 2, 2000)
    tokens[2] = -1
    _check(x, tokens, 6, got)
    sv.close()


def test_score_after_and_before_sample(etc):
    """Sampling and scores share a handle's workspace: long rows of both in turn, twice the same."""
    vocab, rows = 60000, 7
    x, tokens = _logits(8, rows, vocab), _tokens(9, rows, vocab)
    sv = etc.Serving(ref.shape(vocab=vocab), max_seqs=rows, max_tokens=rows, max_kv_len=1)
    dev, u = x.cuda(), torch.full((rows,), 0.37, device="cuda")
    first = None
    for _ in range(3):
        token, lp = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
        sv.sample(dev, u, token, logprob_out=lp)
        got = _run(etc, x, tokens, 11, serving=sv)
        _check(x, tokens, 11, got)
        again = {"token": token.cpu().numpy(), "lp": lp.cpu().numpy(), **got}
        first = first or again
        assert all(np.array_equal(first[k], again[k]) for k in first)
        drawn = _run(etc, x, token.cpu().numpy(), 0, serving=sv)["logprob"]
        assert np.allclose(drawn, again["lp"], atol=2.0 ** -16)          # without filters both are the same share
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 300, 16000, 40000])
def test_score_large_logits(etc, vocab, dtype):
    """Logits far from zero, neighbours in their type: from about 2^27 on those differ by more than an exponential tells apart, and a multiple of
    one by 1 / ln 2 is rounded by as much.  The rounding of a reference, 2^-24 of it and 64 at most where sums count from it (2^30), is what
    sums of p ln p are counted from: their roundings (as in _check) are relative to it too."""
    g = torch.Generator().manual_seed(vocab)
    bits = torch.int32 if dtype == torch.float32 else torch.int16
    rows = []
    for e in (20, 24, 26, 27, 28, 29, 30, 31, 33, 40, 64, 100, 126):
        for m in (1.0, 1.4, 1.96):
            for sign in (1, -1):
                most = torch.tensor([sign * m * 2.0 ** e]).to(dtype).view(bits)
                rows.append((most - sign * torch.randint(0, 40, (vocab,), generator=g).to(bits)).view(dtype))
    for sign in (1, -1):                                 # both sides of 2^30, by parts of a row and mixed
        edge = torch.tensor([sign * 2.0 ** 30]).to(dtype).view(bits)
        for up in ([vocab // 2], [0, vocab - 1], list(range(0, vocab, 3))):
            k = torch.zeros(vocab, dtype=bits)
            k[up] = sign
            rows += [(edge + k).view(dtype), (edge - k).view(dtype)]
    x = torch.stack(rows)
    tokens = torch.where(torch.arange(len(rows)) % 2 == 0, x.double().argmax(1), torch.randint(0, vocab, (len(rows),), generator=g)).numpy()
    got = _run(etc, x, tokens, 9)
    entropy = got["entropy"].copy()
    got["entropy"][:] = 55.0
    _check(x, tokens, 9, got)
    for r in range(len(rows)):
        want = codes.score(x[r].double().numpy(), None, 0)[1]
        off = min(64.0, 1.4427 * 2.0 ** -24 * float(x[r].double().abs().max()))
        assert abs(entropy[r] - want) <= 2.0 ** -17 * (8 + off + want), (r, entropy[r], want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 300, 16000, 40000])
def test_score_is_no_more_than_certain(etc, vocab, dtype):
    """Rows of one likely token, alone or far above the others: a logarithm of a probability is not above 0, whatever was rounded on the way."""
    g = torch.Generator().manual_seed(vocab)
    rows = 64
    tokens = torch.randint(0, vocab, (rows,), generator=g)
    most = torch.randn(rows, generator=g) * torch.tensor([1.0, 30.0, 1e4, 1e8]).repeat(rows // 4)
    most[4], most[9] = 2.5e38, -3e38
    x = torch.full((rows, vocab), -math.inf)
    x[::2] = most[::2, None] - 40 - 3 * torch.rand(rows // 2, vocab, generator=g)
    x = x.scatter(1, tokens[:, None], most[:, None]).to(dtype)
    got = _run(etc, x, tokens.numpy(), 5)
    _check(x, tokens.numpy(), 5, got)
    assert (got["logprob"] <= 0).all() and (got["tops"] <= 0).all() and (got["entropy"] >= 0).all()


def test_score_repeats(etc):
    """The same pointers give the same bits, and so do rows that lie alike in memory (their first elements' places modulo 16 bytes)."""
    for vocab, dtype, rows, stride in ((30001, torch.bfloat16, 24, 0), (30001, torch.float32, 9, 0), (30001, torch.bfloat16, 9, 7), (1003, torch.float32, 530, 0)):
        one = _logits(vocab, 1, vocab, dtype)
        x = one.repeat(rows, 1)
        tokens = np.full(rows, 77)
        sv = etc.Serving(ref.shape(vocab=vocab), max_seqs=rows if rows <= 1024 else 1024, max_tokens=rows, max_kv_len=1)
        first = _run(etc, x, tokens, 7, stride=stride, serving=sv)
        again = _run(etc, x, tokens, 7, stride=stride, serving=sv)
        assert all(np.array_equal(first[k], again[k]) for k in first)
        _check(x, tokens, 7, first, rows=range(0, rows, 5))
        alike = 16 // dtype.itemsize // math.gcd(vocab + stride, 16 // dtype.itemsize)
        for r in range(rows - alike):
            assert all(np.array_equal(first[k][r], first[k][r + alike]) for k in first), r
        assert sv.read_error() == (0, 0, 0, 0)
        sv.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,top", [(513, 128256, 5), (600, 70001, 64), (520, 16385, 0)])
def test_score_long_rows_not_cut(etc, dtype, rows, vocab, top):
    """More rows than are cut: a workgroup goes through a long row, its threshold found again many times."""
    x, tokens = _logits(rows, rows, vocab, dtype), _tokens(rows, rows, vocab)
    n = torch.arange(vocab).float() / vocab
    x[0], x[1], x[2], x[3] = 10 * n, -10 * n, 2.0, (7 * n).round()          # rising, falling, flat, ties that rise
    x[4], x[4, -9:], x[5, ::2] = -math.inf, 1.0, math.nan
    _check(x, tokens, top, _run(etc, x, tokens, top), rows=[*range(7), *range(7, rows, 40), rows - 1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,top", [(300, 20001, 64), (512, 16384, 9), (40, 128256, 64), (513, 20001, 5)])
def test_score_more_rows_than_sequences(etc, dtype, rows, vocab, top):
    """The workspace of the smallest handle, and scores of many rows in it."""
    x, tokens = _logits(rows, rows, vocab, dtype), _tokens(rows, rows, vocab)
    _check(x, tokens, top, _run(etc, x, tokens, top, max_seqs=1), rows=[*range(0, rows, 20), rows - 1])
