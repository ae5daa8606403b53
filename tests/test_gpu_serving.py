"""Serving operators on the GPU, one by one, against their plain 64-bit forms on the CPU (tests/serving_ref.py)."""
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


# ---- tables -----------------------------------------------------------------------------------------------------------
def _tables_call(etc, kv, new, page=16, rows=None, cols=None, free=None, alias=False, csr=True, ids_cap=None, max_tokens=None):
    s = ref.shape(page=page)
    rows = sum(new) + 2 if rows is None else rows
    rng = np.random.default_rng(len(kv) * 7 + sum(new))
    need = [ref.pages_needed(k + n, page) for k, n in zip(kv, new)]
    cols = max(need + [1]) + 1 if cols is None else cols
    ids = rng.permutation(sum(need) + 9)
    table, at = np.full((len(kv), cols), -7, np.int32), 0
    for b, k in enumerate(kv):
        n = min(ref.pages_needed(k, page), cols)
        table[b, :n] = ids[at:at + n]
        at += n
    free = list(ids[at:]) if free is None else free
    sv = etc.Serving(s, max_seqs=len(kv), max_tokens=max(1, rows if max_tokens is None else max_tokens), max_kv_len=1 << 20)
    e = lambda n: torch.full((n,), 12345, dtype=torch.int32, device="cuda")        # noqa: E731
    io = {"kv": i32(kv), "new": i32(new), "table": i32(table), "free": i32(free + [0] * 4), "count": i32([len(free)])}
    out = {"q_indptr": e(len(kv) + 1), "slots": e(rows), "positions": e(rows), "status": e(1)}
    more = {"total_len": io["kv"] if alias else e(len(kv)), "free_count_out": None if alias else e(1)}
    if csr:
        more.update(page_indptr=e(len(kv) + 1), page_ids=e(sum(need) if ids_cap is None else ids_cap))
    sv.tables(io["kv"], io["new"], io["table"], io["free"], io["count"], **out, **more)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in {**out, **more}.items() if v is not None}
    got["free_count"] = (io["count"] if alias else more["free_count_out"]).cpu().numpy()
    got["block_table"] = io["table"].cpu().numpy()
    got.pop("free_count_out", None)
    sv.close()
    return got, table, free, rows


@pytest.mark.parametrize("page", [1, 2, 16, 256])
@pytest.mark.parametrize("kv,new", [([0], [1]), ([5], [0]), ([15, 16, 17, 0], [1, 1, 0, 40]), ([0] * 3, [0] * 3),
                                    (list(range(0, 1024 * 3, 3)), [1] * 1024), ([300, 0, 31], [5000, 3000, 1])])
@pytest.mark.parametrize("alias", [False, True])
def test_tables(etc, kv, new, page, alias):
    got, table, free, rows = _tables_call(etc, kv, new, page=page, alias=alias)
    want = ref.tables(kv, new, table, free, page, rows)
    for name, w in want.items():
        assert np.array_equal(got[name], np.asarray(w)), name


@pytest.mark.parametrize("why", ["pages", "rows", "cols", "negative", "long", "ids"])
@pytest.mark.parametrize("many", [False, True])
def test_tables_are_all_or_nothing(etc, why, many):
    kv, new = [20, 3, 40], [30, 1, 0]
    if many:                                              # several workgroups
        kv, new = kv + [7] * 200, new + [25] * 200
    kw, status = {}, -1
    rows = sum(new) + 2
    if why == "pages":
        kw["free"], status = [3, 4], sum(ref.pages_needed(k + n, 16) - ref.pages_needed(k, 16) for k, n in zip(kv, new)) - 2
        if status <= 0:
            kw["free"], status = [], status + 2
    elif why == "rows":
        rows = sum(new) - 1
    elif why == "cols":
        kw["cols"] = 3
    elif why == "negative":
        new[1] = -1
    elif why == "long":
        kv[2] = (1 << 20) + 1
        kw["cols"] = 4
    else:
        kw["ids_cap"] = 5
    if why == "long":
        kw["free"] = list(range(500))
    got, table, free, rows = _tables_call(etc, kv, new, rows=rows, **kw)
    assert got["status"][0] == status
    assert np.array_equal(got["block_table"], table) and got["free_count"][0] == len(free)
    assert (got["slots"] == -1).all() and (got["positions"] == 0).all() and (got["q_indptr"] == 0).all()
    assert (got["page_indptr"] == 0).all() and (got["page_ids"] == 12345).all() and np.array_equal(got["total_len"], kv)


# ---- append -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (1, 1, 128), (6, 2, 128), (32, 8, 128), (40, 8, 64), (7, 7, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("qk_norm", [False, True])
@pytest.mark.parametrize("tokens,page", [(1, 16), (37, 1), (130, 64)])
def test_append(etc, nq, nkv, d, dtype, qk_norm, tokens, page):
    s = ref.shape(nq, nkv, d, page=page, qk_norm=qk_norm, theta=1e6)
    gap = 16                                              # q, k, v as parts of wider rows
    qkv = randn(1, tokens, (nq + 2 * nkv) * d + gap, dtype=dtype) * 3
    gains = (1 + randn(2, 2, d)).bfloat16() if qk_norm else None
    n_pages = ref.pages_needed(tokens, page) + 2
    rng = np.random.default_rng(3)
    slots = rng.permutation(n_pages * page)[:tokens].astype(np.int32)
    slots[rng.random(tokens) < 0.2] = -1                  # padding among the rows
    pos = rng.integers(0, 1 << 20, tokens).astype(np.int32)
    pos[0] = 0
    k0, v0, q0 = randn(4, n_pages, page, nkv, d), randn(5, n_pages, page, nkv, d), randn(6, tokens, nq, d)
    dev = [t.cuda() for t in (qkv, k0, v0, q0)]
    sv = etc.Serving(s, max_seqs=1, max_tokens=tokens, max_kv_len=1 << 20)
    a, b = nq * d, (nq + nkv) * d
    g = (None, None) if gains is None else (gains[0].cuda(), gains[1].cuda())
    sv.append(dev[0][:, :a], dev[0][:, a:b], dev[0][:, b:b + nkv * d], i32(pos), i32(slots), dev[3], dev[1], dev[2], gq=g[0], gk=g[1])
    torch.cuda.synchronize()
    live = slots >= 0
    x = qkv[:, :(nq + 2 * nkv) * d].view(tokens, nq + 2 * nkv, d)
    for got, old, heads, gain in ((dev[3], q0, slice(0, nq), 0), (dev[1].view(-1, nkv, d), k0.view(-1, nkv, d), slice(nq, nq + nkv), 1)):
        want, size = ref.rotate(s, x[:, heads], pos, None if gains is None else gains[gain])
        at = torch.as_tensor(np.nonzero(live)[0] if gain == 0 else slots[live].astype(np.int64))
        full = old.double().clone()
        full[at] = want[torch.as_tensor(live)]
        # one rounding to bf16; norm factor, angle (reduced in fp64), sine and cosine in fp32, the last two by instruction: 2^-16 of a + b
        tol = torch.zeros_like(full)
        tol[at] = (2.0 ** -8 * want.abs() + 2.0 ** -16 * size)[torch.as_tensor(live)]
        assert bool(((got.cpu().double() - full).abs() <= tol).all())
    vv = v0.clone().view(-1, nkv, d)
    vv[torch.as_tensor(slots[live].astype(np.int64))] = x[torch.as_tensor(live), nq + nkv:].bfloat16()
    assert torch.equal(dev[2].cpu().view(-1, nkv, d), vv)
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()


def test_append_in_place_and_bad_slots(etc):
    s = ref.shape(4, 2, 64, page=16)
    q, k, v = randn(1, 9, 256).cuda(), randn(2, 9, 128).cuda(), randn(3, 9, 128).cuda()
    pools = [torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    sv = etc.Serving(s, max_seqs=1, max_tokens=9, max_kv_len=100)
    out = torch.zeros(9, 4, 64, dtype=torch.bfloat16, device="cuda")
    slots = np.arange(9)
    sv.append(q, k, v, i32(np.arange(9)), i32(slots), out, pools[0], pools[1])
    bad = slots.copy()
    bad[[2, 5]] = [32, 1 << 30]                          # outside the pool: the rows are left out, the next call says so
    qq = q.clone()
    sv.append(qq, k, v, i32(np.arange(9)), i32(bad), qq.view(9, 4, 64), pools[2], pools[3])
    torch.cuda.synchronize()
    keep = [0, 1, 3, 4, 6, 7, 8]
    assert torch.equal(qq.view(9, 4, 64)[keep], out[keep]) and torch.equal(qq[[2, 5]], q[[2, 5]])
    assert torch.equal(pools[2].view(32, 2, 64)[keep], pools[0].view(32, 2, 64)[keep]) and bool((pools[2].view(32, 2, 64)[[2, 5]] == 0).all())
    with pytest.raises(etc.EtcError, match="slot outside the pool"):
        sv.append(q, k, v, i32(np.arange(9)), i32(slots), out, pools[0], pools[1])
    sv.append(q, k, v, i32(np.arange(9)), i32(slots), out, pools[0], pools[1])      # reported once, then usable
    torch.cuda.synchronize()
    assert sv.read_error()[0] == 0
    sv.close()


# ---- attention ----------------------------------------------------------------------------------------------------------
def _attention(etc, s, kv, new, seed=0, pad=0, poison=None, sigma=1.0, table_pad=0):
    table, n_pages = ref.paged([a + b for a, b in zip(kv, new)], s.page, seed)
    q_indptr = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
    rows = int(q_indptr[-1]) + pad
    q = (randn(seed + 1, rows, s.nq, s.d) * sigma).bfloat16()
    k, v = randn(seed + 2, n_pages, s.page, s.nkv, s.d), randn(seed + 3, n_pages, s.page, s.nkv, s.d)
    if poison is not None:
        poison(k, v, table, kv, new)
    out = torch.full((rows, s.nq, s.d), 7.0, dtype=torch.bfloat16, device="cuda")
    wide = np.full((table.shape[0], table.shape[1] + table_pad), -1, np.int32)
    wide[:, :table.shape[1]] = table
    sv = etc.Serving(s, max_seqs=len(kv), max_tokens=max(rows, 1), max_kv_len=max(a + b for a, b in zip(kv, new)) + 1)
    sv.attention(q.cuda(), out, i32(q_indptr), i32(kv), i32(wide)[:, :table.shape[1]], k.cuda(), v.cuda())
    torch.cuda.synchronize()
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    got = out.cpu()
    n = int(q_indptr[-1])
    assert bool((got[n:] == 7.0).all())                  # rows behind the last sequence
    want, size = ref.attention(s, q, k, v, q_indptr, kv, table)
    ref.check_attention(got[:n], want[:n], size[:n])
    return got


SHAPES = [(4, 2, 64), (32, 8, 128), (8, 1, 128), (2, 2, 128), (5, 1, 64), (12, 4, 128)]


@pytest.mark.parametrize("nq,nkv,d", SHAPES)
@pytest.mark.parametrize("kv,new", [([0], [1]), ([7], [1]), ([63, 64, 65], [1, 1, 1]), ([0, 130, 20], [70, 0, 33]), ([500], [3]),
                                    ([200, 0, 1, 31], [1, 129, 64, 2]), ([1500, 3], [40, 1])])
def test_attention(etc, nq, nkv, d, kv, new):
    _attention(etc, ref.shape(nq, nkv, d), kv, new, pad=3, table_pad=2)


@pytest.mark.parametrize("page", [1, 2, 8, 128, 1024])
def test_attention_page_sizes(etc, page):
    _attention(etc, ref.shape(8, 2, 128, page=page), [0, 100, 1027], [35, 1, 70])


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (32, 8, 128), (8, 1, 128)])
@pytest.mark.parametrize("kv,new", [([20000], [1]), ([9000], [9]), ([0], [700]), ([6000, 0, 50, 3000], [1, 300, 1, 1]), ([1] * 40 + [12000], [1] * 41),
                                    ([4095, 4096, 4097], [33, 32, 31])])
def test_attention_keys_in_parts(etc, nq, nkv, d, kv, new):
    """Long contexts of few rows, and long chunks: the keys of an item are cut into pieces, short blocks into fewer than long ones."""
    _attention(etc, ref.shape(nq, nkv, d), kv, new, seed=7)


def test_attention_is_the_same_every_time(etc):
    """Partial results are joined in the order of the keys, whoever comes last; the workspace is as it was after a call."""
    s = ref.shape(8, 2, 128)
    table, n_pages = ref.paged([5000, 700], 16, 1)
    q, k, v = randn(1, 45, 8, 128).cuda(), randn(2, n_pages, 16, 2, 128).cuda(), randn(3, n_pages, 16, 2, 128).cuda()
    out, qi, kv, t = torch.zeros_like(q), i32([0, 5, 45]), i32([4995, 660]), i32(table)
    sv = etc.Serving(s, max_seqs=2, max_tokens=45, max_kv_len=5000)
    sv.attention(q, out, qi, kv, t, k, v)
    for _ in range(20):
        again = torch.full_like(q, 3.0)
        sv.attention(q, again, qi, kv, t, k, v)
        assert torch.equal(again, out)
    sv.close()


def test_attention_many_sequences(etc):
    rng = np.random.default_rng(1)
    new = rng.integers(0, 4, 700).tolist()
    _attention(etc, ref.shape(2, 1, 64), rng.integers(0, 90, 700).tolist(), new, pad=1)


def test_attention_most_sequences(etc):
    rng = np.random.default_rng(2)
    new = rng.choice([0, 1, 1, 1, 2, 30], 1024).tolist()
    _attention(etc, ref.shape(4, 2, 64, page=8), rng.integers(0, 300, 1024).tolist(), new)


def test_attention_few_and_many_rows_together(etc):
    """More pieces than workgroups, of sequences of a few tokens and of prompts: in another order than the sequences'."""
    rng = np.random.default_rng(3)
    _attention(etc, ref.shape(8, 2, 64, page=8), rng.integers(0, 200, 700).tolist(), rng.choice([0, 1, 1, 2, 40], 700).tolist(), pad=2)
    _attention(etc, ref.shape(8, 8, 64), rng.integers(10, 3000, 40).tolist(), [1] * 9 + [150] + [3] * 20 + [300, 0] + [1] * 8)
    _attention(etc, ref.shape(4, 4, 128), rng.integers(0, 400, 70).tolist(), [80 + i for i in range(70)])


@pytest.mark.parametrize("new", [1, 70])
def test_attention_more_pages_than_a_window(etc, new):
    """Pages of one token, and as many sequences as workgroups take without cutting their keys: page ids come 1024 at a time."""
    _attention(etc, ref.shape(8, 8, 64, page=1), [1600] * 33, [new] * 33)
    _attention(etc, ref.shape(8, 8, 64, page=1), [1023 + 5 * i for i in range(32)], [new] * 32)


def test_far_pages(etc):
    """Pools of more than 4 GiB: append and attention at their end."""
    s = ref.shape(16, 8, 128, page=16)
    n_pages, used = 150000, 12
    pools = [torch.zeros(n_pages, 16, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert pools[0].numel() * 2 > 1 << 32
    for i, p in enumerate(pools):
        p[-used:] = randn(i, used, 16, 8, 128).cuda()
    table = np.arange(n_pages - used, n_pages, dtype=np.int32)[::-1].copy().reshape(2, used // 2)
    kv, new = [60, 3], [30, 80]
    slots = [int(table[b, p // 16]) * 16 + p % 16 for b in range(2) for p in range(kv[b], kv[b] + new[b])]
    pos = [p for b in range(2) for p in range(kv[b], kv[b] + new[b])]
    rows = randn(5, 110, 32 * 128).cuda().split([16 * 128, 8 * 128, 8 * 128], 1)
    q, out = torch.zeros(110, 16, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(110, 16, 128, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=2, max_tokens=110, max_kv_len=96)
    sv.append(*rows, i32(pos), i32(slots), q, *pools)
    sv.attention(q, out, i32([0, 30, 110]), i32(kv), i32(table), *pools)
    torch.cuda.synchronize()
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    near = [p[-used:].cpu() for p in pools]
    assert torch.equal(near[1].view(-1, 8, 128)[torch.as_tensor(slots) - (n_pages - used) * 16], rows[2].cpu().reshape(-1, 8, 128))
    want, size = ref.attention(s, q, *near, [0, 30, 110], kv, table - (n_pages - used))
    ref.check_attention(out, want, size)
    assert not any(bool(p[:-used].any()) for p in pools)


def test_attention_large_scores(etc):
    _attention(etc, ref.shape(4, 2, 64), [300, 0], [20, 65], sigma=12.0)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_attention_what_a_row_does_not_see(etc, value):
    """NaN and infinities in later tokens of the chunk, behind the last token of a page and in pages of nobody."""
    def poison(k, v, table, kv, new):
        s_page = k.shape[1]
        used = set()
        for b, (a, n) in enumerate(zip(kv, new)):
            used |= {int(table[b, p]) for p in range(ref.pages_needed(a + n, s_page))}
            last = a + n - 1
            page = int(table[b, last // s_page])
            for pool in (k, v):
                pool[page, last % s_page + 1:] = value
            if n > 3:                                     # the last two tokens of the chunk: their own rows see them
                for t in (last - 1, last):
                    v[int(table[b, t // s_page]), t % s_page, :, ::3] = value
        for p in set(range(k.shape[0])) - used:
            k[p], v[p] = value, value
    _attention(etc, ref.shape(8, 2, 128), [5, 700, 0, 129], [40, 1, 130, 5], poison=poison)


def test_attention_mixed_infinities(etc):
    def poison(k, v, table, kv, new):
        for t, val in ((10, math.inf), (20, -math.inf), (30, math.nan)):
            v[int(table[0, t // 16]), t % 16, :, 3] = val
            v[int(table[0, (t + 1) // 16]), (t + 1) % 16, :, t] = val
    _attention(etc, ref.shape(4, 2, 64), [0], [50], poison=poison)


def test_attention_bad_pages_and_lengths(etc):
    s = ref.shape(4, 2, 64)
    q = randn(1, 3, 4, 64).cuda()
    k, v = randn(2, 6, 16, 2, 64).cuda(), randn(3, 6, 16, 2, 64).cuda()
    table = np.array([[0, 1], [2, 1 << 30], [4, 5]], np.int32)
    sv = etc.Serving(s, max_seqs=3, max_tokens=3, max_kv_len=32)
    call = lambda t, kv, qi=(0, 1, 2, 3): sv.attention(q, out, i32(qi), i32(kv), i32(t), k, v)      # noqa: E731
    out = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    good = torch.zeros_like(out)
    sv.attention(q, good, i32([0, 1, 2, 3]), i32([20, 10, 31]), i32(table), k, v)      # page 1 of sequence 1 is not needed
    torch.cuda.synchronize()
    assert sv.read_error()[0] == 0
    for t, kv, qi, b, code in ((table, [20, 20, 31], (0, 1, 2, 3), 1, 3), (-table, [20, 10, 31], (0, 1, 2, 3), None, 3),
                               (table, [20, 10, 32], (0, 1, 2, 3), 2, 2), (table, [20, -1, 31], (0, 1, 2, 3), 1, 2),
                               (table, [20, 10, 31], (0, 1, 2, 9), 2, 2), (table, [20, 10, 31], (0, 3, 1, 3), 1, 2), (table, [20, 10, 31], (0, 2, 1, 3), 1, 2)):
        out.zero_()
        call(t, kv, qi)
        torch.cuda.synchronize()
        word = sv.read_error()
        assert word[0] == code and word[1] == 3 and (b is None or word[2] in (b, 3))
        if b is not None and qi == (0, 1, 2, 3):
            keep = [x for x in range(3) if x != b]
            assert torch.equal(out[keep], good[keep])
            if code == 2:
                assert bool((out[b] == 0).all())
    sv.close()


# ---- sampling -----------------------------------------------------------------------------------------------------------
def _sample(etc, x, u, stride_pad=0, **settings):
    """Checks every row, and returns how many rows stood next to a border (gap below 1e-7) and were not compared."""
    rows, vocab = x.shape
    sv = etc.Serving(ref.shape(vocab=vocab), max_seqs=rows, max_tokens=1, max_kv_len=1)
    wide = torch.full((rows, vocab + stride_pad), 1e30, dtype=x.dtype)
    wide[:, :vocab] = x
    tok, kept = (torch.full((rows,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    lp = torch.zeros(rows, device="cuda")
    dev = {k: torch.as_tensor(np.asarray(v, np.int32 if k == "top_k" else np.float32)).cuda() for k, v in settings.items()}
    sv.sample(wide.cuda()[:, :vocab], torch.as_tensor(np.asarray(u, np.float32)).cuda(), tok, logprob_out=lp, kept_out=kept, **dev)
    torch.cuda.synchronize()
    sv.close()
    skipped = 0
    xs = x.double().numpy()
    for r in range(rows):
        own = {k: float(np.float32(v[r])) if k != "top_k" else int(v[r]) for k, v in settings.items()}
        t, p, n, gap = ref.sample_row(xs[r], float(np.float32(u[r])), **own)
        if gap < 1e-7:                                    # a weight is off by 2^-34 of it and half of 2^-35: 128256 of them by 6 sigma = 2e-8 of a sum
            skipped += 1
            continue
        assert int(tok[r]) == t and int(kept[r]) == n, (r, own, int(tok[r]), t, int(kept[r]), n)
        # fp32 rounding of the result; the sum of weights is at least 1, each of them off by half of 2^-35 and 2^-34 of itself at most
        assert abs(float(lp[r]) - p) <= 2.0 ** -24 * abs(p) + 2.0 ** -36 * vocab + 2.0 ** -34 or float(lp[r]) == p
    return skipped


def _logits(seed, rows, vocab, dtype, sigma=2.5):
    return (randn(seed, rows, vocab, dtype=torch.float32) * sigma).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 63, 1024, 1025, 5000, 128256])
def test_sample_settings(etc, dtype, vocab):
    rng = np.random.default_rng(vocab)
    rows = 24
    x = _logits(vocab, rows, vocab, dtype)
    kw = dict(temperature=rng.choice([0.0, 0.3, 1.0, 1.7], rows), top_k=rng.choice([0, 1, 2, 7, 50, 3000, 1 << 30, -3], rows),
              top_p=rng.choice([1.0, 0.999, 0.9, 0.3, 0.0, -1.0, 2.0], rows), min_p=rng.choice([0.0, 0.0, 0.01, 0.3, 1.0, 1.5, -1.0], rows))
    u = rng.random(rows, np.float32)
    assert _sample(etc, x, u, stride_pad=3, **kw) < rows // 2
    for one in kw:
        assert _sample(etc, x, u, **{one: kw[one]}) < rows // 2
    _sample(etc, x, u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sample_ties_and_flat_rows(etc, dtype):
    """Equal logits: ids in ascending order; a flat row keeps any count exactly, and the draw walks it."""
    vocab = 4099
    x = torch.zeros(12, vocab, dtype=dtype)
    x[4:8] = torch.arange(vocab).remainder(3).to(dtype)
    x[8:, 100:200] = 2
    x[:, 7] = -0.0                                        # equal to 0
    u = [0.0, 0.2501, 0.7503, 0.99999] * 3
    _sample(etc, x, u)
    _sample(etc, x, u, top_k=[1, 2, 1000, 4099] * 3)
    _sample(etc, x, u, top_k=[1500] * 12, top_p=[0.50001] * 12)
    _sample(etc, x, u, min_p=[0.9] * 12)
    _sample(etc, x, u, temperature=[0.0] * 12)


@pytest.mark.parametrize("vocab", [16382, 16383, 16384, 16385])
def test_sample_longest_rows_of_one_launch(etc, vocab):
    """All tokens in one bin, each with the largest weight: counts and weights of a bin share a word."""
    x = torch.zeros(4, vocab)
    x[1, 5:] = -60.0                                      # beyond the bins
    x[2] = _logits(2, 1, vocab, torch.float32)[0]
    x[3, ::2] = 1.0
    u = [0.50001, 0.3, 0.7, 0.99]
    _sample(etc, x, u)
    _sample(etc, x, u, top_k=[vocab - 1, 9000, 9000, 8100], top_p=[0.75001] * 4)


def test_sample_a_slice_of_equal_logits(etc):
    """The largest vocabulary in as many slices as there are with 4 rows: the first tokens all weigh as much as the largest."""
    vocab = 1 << 20
    x = _logits(9, 4, vocab, torch.float32, sigma=1.0) - 12.0
    x[:, :16384] = 0.0
    x[2, 16000:] -= 5.0
    u = [0.2, 0.9999, 0.9995, 0.99999]
    assert _sample(etc, x, u) < 4
    _sample(etc, x, u, top_p=[0.5, 0.99999, 0.999, 1.0], top_k=[0, 0, 300000, 17000])


@pytest.mark.parametrize("rows", [128, 129])
def test_sample_rows_with_and_without_shares(etc, rows):
    """Two workgroups to a row, and one; rows that need none, and flat ones whose tokens fill no list, among them."""
    vocab = 33001
    x = _logits(rows, rows, vocab, torch.bfloat16)
    x[3], x[77], x[100] = -math.inf, 0.25, math.nan
    x[5, 40:] = -math.inf
    x[9, 30000] = math.inf
    rng = np.random.default_rng(rows)
    kw = dict(temperature=rng.choice([0.0, 0.5, 1.0, 2.0], rows), top_k=rng.choice([0, 1, 40, 20000], rows), top_p=rng.choice([1.0, 0.9, 0.2], rows),
              min_p=rng.choice([0.0, 0.05], rows))
    for _ in range(2):
        assert _sample(etc, x, rng.random(rows, np.float32), **kw) < rows // 2


def test_sample_banned_and_infinite(etc):
    vocab = 3001
    x = _logits(5, 10, vocab, torch.float32)
    x[0] = -math.inf                                      # nothing left
    x[1] = math.nan
    x[2, :] = -math.inf
    x[2, 2999] = -3e38                                    # one token left
    x[3, ::2] = -math.inf
    x[4, ::3] = math.nan
    x[5, [17, 600]] = math.inf                            # infinite: those alone
    x[6] = torch.finfo(torch.float32).min                 # the type's lowest value is a logit like any other
    x[7, :] = torch.finfo(torch.float32).min
    x[7, 5] = 3e38
    x[8, 0] = math.inf
    x[9] = -math.inf
    x[9, 0] = math.nan
    u = np.linspace(0, 0.95, 10)
    for kw in ({}, {"top_k": [3] * 10}, {"top_p": [0.5001] * 10}, {"min_p": [0.3] * 10}, {"temperature": [0.0] * 10},
               {"temperature": [math.inf] * 10}, {"temperature": [1e-30] * 10}):
        _sample(etc, x, u, **kw)


def test_sample_nan_settings_and_u_out_of_range(etc):
    x = _logits(3, 4, 500, torch.float32)
    nan = [math.nan] * 4
    sv = etc.Serving(ref.shape(vocab=500), max_seqs=4, max_tokens=1, max_kv_len=1)
    tok, want = (torch.zeros(4, dtype=torch.int32, device="cuda") for _ in range(2))
    f = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")        # noqa: E731
    u = f([0.1, 0.4, 0.6, 0.9])
    sv.sample(x.cuda(), u, tok, top_p=f(nan), min_p=f(nan))
    sv.sample(x.cuda(), u, want)
    torch.cuda.synchronize()
    assert torch.equal(tok, want)
    sv.sample(x.cuda(), u, tok, temperature=f(nan))
    sv.sample(x.cuda(), u, want, temperature=f([0.0] * 4))
    torch.cuda.synchronize()
    assert torch.equal(tok, want) and torch.equal(want.cpu().long(), x.argmax(-1))
    sv.sample(x.cuda(), f([-1.0, math.nan, 1.0, 5.0]), tok)
    order = x.sort(dim=-1, descending=True, stable=True).indices
    torch.cuda.synchronize()
    assert tok[0] == order[0, 0] and tok[1] == order[1, 0]            # below the range and NaN: as 0
    assert tok[2] == order[2, -1] and tok[3] == order[3, -1]          # above: the last that is kept
    sv.close()
