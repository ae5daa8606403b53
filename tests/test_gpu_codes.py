"""The paged cache of 8-bit codes on the GPU: append and attention, one by one, against their plain 64-bit forms on the CPU."""
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


# ---- append -----------------------------------------------------------------------------------------------------------
# How far fp32 leaves the values that are rounded to codes, relative to the sizes of the two products that a rotated element is the sum of:
# two products and a sum (2^-22), sine and cosine of 2 units in the last place of an angle rounded to fp32 (2^-21), and with norms a sum of D squares in
# chains of at most 20 additions, its root, division and two products (2^-19.5).  The same for queries, in front of their own rounding.
FP32 = 2.0 ** -19


def _slots(rng, new, kv, page, extra=2):
    """Slots and positions of sequences' new tokens in pages of their own, as tables() gives them, with padding rows between."""
    need = [ref.pages_needed(k + n, page) - k // page for k, n in zip(kv, new)]
    n_pages = sum(need) + extra
    ids, slots, pos, at = rng.permutation(n_pages), [], [], 0
    for k, n, m in zip(kv, new, need):
        for t in range(k, k + n):
            slots.append(int(ids[at + t // page - k // page]) * page + t % page)
            pos.append(t)
        at += m
        pad = int(rng.integers(0, 3))
        slots += [-1] * pad
        pos += [0] * pad
    return np.asarray(slots, np.int32), np.asarray(pos, np.int32), n_pages


def _append(etc, s, kv, new, dtype, seed=1, scale=1.0, change=None, repeat=1):
    rng = np.random.default_rng(seed)
    slots, pos, n_pages = _slots(rng, new, kv, s.page)
    rows, gap = len(slots), 16
    qkv = randn(seed, rows, (s.nq + 2 * s.nkv) * s.d + gap, dtype=torch.float32)
    qkv *= scale * torch.exp2(torch.as_tensor(rng.integers(-2, 3, (rows, 1))).float())       # runs of different sizes
    if change is not None:
        change(qkv, s)
    qkv = qkv.to(dtype)
    gains = (1 + randn(seed + 1, 2, s.d)).bfloat16() if s.qk_norm else None
    (k0, ks0), (v0, vs0) = codes.pools(seed + 2, n_pages, s.page, s.nkv, s.d), codes.pools(seed + 3, n_pages, s.page, s.nkv, s.d)
    q0 = randn(seed + 4, rows, s.nq, s.d)
    x, q, k, ks, v, vs = [t.cuda() for t in (qkv, q0, k0, ks0, v0, vs0)]
    a, b = s.nq * s.d, (s.nq + s.nkv) * s.d
    g = (None, None) if gains is None else (gains[0].cuda(), gains[1].cuda())
    sv = etc.Serving(s, max_seqs=max(1, len(kv)), max_tokens=max(1, rows), max_kv_len=1 << 20)
    for _ in range(repeat):
        sv.append_codes(x[:, :a], x[:, a:b], x[:, b:b + s.nkv * s.d], i32(pos), i32(slots), q, k, v, ks, vs, gq=g[0], gk=g[1])
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    heads = qkv[:, :b + s.nkv * s.d].view(rows, -1, s.d)
    live = torch.as_tensor(slots >= 0)
    want, size = ref.rotate(s, heads[:, :s.nq], pos, None if gains is None else gains[0])
    full, tol = q0.double().clone(), torch.zeros(rows, s.nq, s.d, dtype=torch.float64)
    full[live], tol[live] = want[live], (2.0 ** -8 * want.abs() + FP32 * size)[live]
    got = q.cpu().double()
    fine = torch.isfinite(full)
    assert bool((torch.isfinite(got) | ~fine).all()) and bool(((got - full).abs() <= tol)[fine].all())
    want, size = ref.rotate(s, heads[:, s.nq:s.nq + s.nkv], pos, None if gains is None else gains[1])
    codes.check_append(s.page, slots, want, torch.nan_to_num(FP32 * size, nan=0.0, posinf=0.0), k0, ks0, k, ks)
    vv = heads[:, s.nq + s.nkv:].double()
    codes.check_append(s.page, slots, vv, torch.zeros_like(vv), v0, vs0, v, vs)


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (1, 1, 128), (6, 2, 128), (32, 8, 128), (40, 8, 64), (7, 7, 64), (9, 9, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("qk_norm", [False, True])
@pytest.mark.parametrize("kv,new,page", [([5], [1], 16), ([0, 15, 16, 30, 7], [1, 1, 1, 40, 12], 16), ([3, 0], [37, 2], 1), ([0, 70, 200], [130, 9, 100], 64)])
def test_append(etc, nq, nkv, d, dtype, qk_norm, kv, new, page):
    _append(etc, ref.shape(nq, nkv, d, page=page, qk_norm=qk_norm, theta=1e6), kv, new, dtype)


@pytest.mark.parametrize("page", [2, 4, 8, 32, 128, 1024])
def test_append_pages(etc, page):
    _append(etc, ref.shape(4, 2, 128, page=page), [0, page - 1, 3 * page, 5 * page + page // 2], [2 * page + 1, 2, 1, page], torch.bfloat16, seed=page)


def test_append_many_rows(etc):
    """Workgroups that look for runs in several rows, runs that go on behind them."""
    rng = np.random.default_rng(0)
    for n, seed in ((300, 5), (60, 6)):
        _append(etc, ref.shape(4, 2, 64), [int(x) for x in rng.integers(0, 5000, n)], [int(x) for x in rng.integers(0, 70, n)], torch.bfloat16, seed=seed)


@pytest.mark.parametrize("scale", [1e-30, 2.0 ** -40, 1e-8, 300.0, 1e30])
def test_append_sizes(etc, scale):
    """Scales up and down to their ends."""
    _append(etc, ref.shape(4, 2, 64), [0, 5, 31], [20, 3, 1], torch.float32, scale=scale)


@pytest.mark.parametrize("page,left_out", [(16, 0.3), (64, 0.7), (256, 0.95)])
def test_append_rows_left_out_between(etc, page, left_out):
    """A page's rows with others between them that have no slot, hundreds of them too."""
    rng = np.random.default_rng(page)
    spread = []
    for slot in list(range(5, 2 * page - 1)) + list(range(3 * page, 3 * page + page // 2)):
        while rng.random() < left_out:
            spread.append(-1)
        spread.append(slot)
    rows = len(spread)
    s = ref.shape(4, 2, 64, page=page)
    x = randn(7, rows, 512, dtype=torch.float32)
    (k0, ks0), (v0, vs0) = codes.pools(1, 5, page, 2, 64), codes.pools(2, 5, page, 2, 64)
    k, ks, v, vs = [t.cuda() for t in (k0, ks0, v0, vs0)]
    q = torch.zeros(rows, 4, 64, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=1, max_tokens=rows, max_kv_len=100000)
    pos = rng.integers(0, 1000, rows)
    sv.append_codes(*x.cuda().split((256, 128, 128), 1), i32(pos), i32(spread), q, k, v, ks, vs)
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    want, size = ref.rotate(s, x[:, 256:384].reshape(rows, 2, 64), pos)
    codes.check_append(page, np.array(spread), want, FP32 * size, k0, ks0, k, ks)
    vv = x[:, 384:].reshape(rows, 2, 64).double()
    codes.check_append(page, np.array(spread), vv, torch.zeros_like(vv), v0, vs0, v, vs)


def test_append_again(etc):
    """The same rows once more: scales stay, so codes do."""
    _append(etc, ref.shape(4, 2, 64), [0, 5, 31], [20, 1, 1], torch.bfloat16, repeat=2)


def test_append_no_numbers(etc):
    def change(x, s):
        b = (s.nq + s.nkv) * s.d
        x[3, b + 5], x[4, b + 70], x[0, b + 1] = math.inf, -math.inf, math.nan
        x[7, s.nq * s.d:] = math.inf                     # a row of nothing else
        x[9, s.nq * s.d + 3], x[2, 7] = math.nan, math.inf
        x[10:, b:] = 0.0
    _append(etc, ref.shape(4, 2, 64), [0, 5, 31], [20, 1, 1], torch.float32, change=change)


def test_append_ends_of_codes(etc):
    """448 times a power of two and its neighbours, ties between codes, what becomes less than the smallest code."""
    def change(x, s):
        b = (s.nq + s.nkv) * s.d
        x[:, b:] = 0.0
        v = x[:, b:b + 2 * s.d]
        v[0, 0], v[0, s.d] = 448.0, 449.0                # the first page: scales 2^0 and 2^1
        v[1, :8] = torch.tensor([17.0, 19.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -10 * 1.001, -2.0 ** -11])
        v[1, s.d:s.d + 4] = torch.tensor([34.0, 38.0, 2.0 ** -9, 464.0])
        v[16, 0], v[16, s.d] = float(np.nextafter(np.float32(448), np.float32(500))), 447.0
    _append(etc, ref.shape(4, 2, 64), [0], [32], torch.float32, change=lambda x, s: (x.mul_(0.01), change(x, s)))


def test_append_refuses_slots(etc):
    s = ref.shape(4, 2, 64)
    q, k, v = (randn(i, 9, n).cuda() for i, n in ((1, 256), (2, 128), (3, 128)))
    (kc, ks), (vc, vs) = codes.pools(4, 2, 16, 2, 64), codes.pools(5, 2, 16, 2, 64)
    dev = [t.cuda() for t in (kc, ks, vc, vs)]
    out = torch.zeros(9, 4, 64, dtype=torch.bfloat16, device="cuda")
    slots = np.array([0, 1, 2, 32, 33, -1, 16, 2 ** 31 - 1, 17], np.int32)
    sv = etc.Serving(s, max_seqs=1, max_tokens=9, max_kv_len=100)
    sv.append_codes(q, k, v, i32(range(9)), i32(slots), out, dev[0], dev[2], dev[1], dev[3])
    code, op, row, slot = sv.read_error()
    assert (code, op) == (1, 5) and (row, slot) in ((3, 32), (7, 2 ** 31 - 1))
    good = np.where((slots >= 0) & (slots < 32), slots, -1)
    vv = v.cpu().double().view(9, 2, 64)
    codes.check_append(16, good, vv, torch.zeros_like(vv), vc, vs, dev[2], dev[3])
    assert not out[[3, 4, 5, 7]].any() and out[[0, 1, 2, 6, 8]].any(-1).all()
    sv.append_codes(q, k, v, i32(range(9)), i32(good), q.view(9, 4, 64), dev[0], dev[2], dev[1], dev[3])      # queries in place
    assert sv.read_error() == (0, 0, 0, 0) and torch.equal(q.view(9, 4, 64)[:3], out[:3])
    sv.close()


# ---- attention ----------------------------------------------------------------------------------------------------------
def _attention(etc, s, kv, new, seed=1, pad=0, spoil=None, check=None, q_change=None, shift=0):
    total = [k + n if n else 0 for k, n in zip(kv, new)]
    table, n_pages = ref.paged(total, s.page, seed)
    (k, ks), (v, vs) = codes.pools(seed + 1, n_pages, s.page, s.nkv, s.d, shift), codes.pools(seed + 2, n_pages, s.page, s.nkv, s.d, shift)
    indptr = np.concatenate(([0], np.cumsum(new)))
    rows = int(indptr[-1]) + pad
    q = randn(seed, rows, s.nq, s.d)
    if q_change is not None:
        q_change(q)
    used = torch.zeros(n_pages, s.page, dtype=torch.bool)
    for b, n in enumerate(total):
        t = np.arange(n)
        used[table[b, t // s.page], t % s.page] = True
    for c in (k, v):                                     # whatever nobody's slots hold
        c.view(torch.uint8)[~used] = 0x7F
    if spoil is not None:
        spoil(k, v, table)
    out = torch.full((rows, s.nq, s.d), 7.0, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=max(1, len(kv)), max_tokens=max(1, rows), max_kv_len=max(total + [1]))
    sv.attention_codes(q.cuda(), out, i32(indptr), i32(kv), i32(table), k.cuda(), v.cuda(), ks.cuda(), vs.cuda())
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    want, size = ref.attention(s, q, codes.values(k, ks), codes.values(v, vs), indptr, kv, table)
    n = int(indptr[-1])
    assert bool((out[n:] == 7.0).all())
    if check is not None:
        return check(out[:n].cpu().double(), want[:n], size[:n], indptr)
    few = max(n * s.nq // s.nkv for n in new) <= 64
    got, want, size = out[:n].cpu().double(), want[:n], size[:n]
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    fine = torch.isfinite(want)
    # The result's rounding (2^-8 of it); scores from q in two codes (2^-21 of the row's largest times the sum of |k|, some 2^-15 of the
    # weight) and in fp32, exponentials and sums: below 2^-12 of the sum of p |v|.  In blocks of many rows probabilities are rounded, 2^-8 each.
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -12 + (0 if few else 2.0 ** -8)) * size + 1e-30
    worst = float(((got - want).abs() / bound)[fine].max()) if n else 0.0
    assert worst <= 1.0, f"worst error / bound {worst:.3f}"


HEADS = [(4, 2, 64), (1, 1, 64), (32, 8, 128), (5, 5, 128), (6, 2, 128), (16, 2, 64), (64, 1, 128)]


@pytest.mark.parametrize("nq,nkv,d", HEADS)
@pytest.mark.parametrize("kv,new", [([0], [1]), ([31, 32, 33, 0], [1, 1, 0, 2]), ([299, 1000, 63], [1, 1, 1]), ([700, 20], [3, 5])])
def test_attention_few_rows(etc, nq, nkv, d, kv, new):
    _attention(etc, ref.shape(nq, nkv, d), kv, new, pad=3)


@pytest.mark.parametrize("nq,nkv,d", HEADS)
@pytest.mark.parametrize("kv,new", [([0], [129]), ([513], [300]), ([0, 777, 64, 5], [77, 1, 130, 64])])
def test_attention_chunks(etc, nq, nkv, d, kv, new):
    _attention(etc, ref.shape(nq, nkv, d), kv, new)


@pytest.mark.parametrize("page", [1, 2, 4, 8, 64, 256])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv,new", [([2100, 90], [1, 1]), ([1500], [260]), ([4500], [70])])
def test_attention_pages(etc, page, d, kv, new):
    """Pages that end inside a step, page ids in several windows."""
    _attention(etc, ref.shape(4, 2, d, page=page), kv, new)


@pytest.mark.parametrize("nq,nkv,d,n", [(64, 32, 64, 8), (32, 16, 128, 16)])
def test_attention_whole_blocks_with_windows(etc, nq, nkv, d, n):
    """Pages of one token, more of them in an uncut piece of a whole block than its window of page ids holds; NaN codes among what no row sees."""
    kv, new = [1090 + 3 * b for b in range(n)], [129 - b for b in range(n)]
    _attention(etc, ref.shape(nq, nkv, d, page=1), kv, new)


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 128), (8, 2, 64)])
def test_attention_long(etc, nq, nkv, d):
    """Keys in many pieces; sequences of few rows among prompts."""
    _attention(etc, ref.shape(nq, nkv, d), [9000], [1])
    _attention(etc, ref.shape(nq, nkv, d), [3000] * 5 + [0, 800], [1, 2, 1, 1, 9, 200, 100])
    _attention(etc, ref.shape(nq, nkv, d), [17000, 5000], [1, 33], seed=5)


@pytest.mark.parametrize("n_seqs", [70, 600])
def test_attention_many_sequences(etc, n_seqs):
    rng = np.random.default_rng(n_seqs)
    kv, new = [int(x) for x in rng.integers(0, 400, n_seqs)], [int(x) for x in rng.integers(0, 3, n_seqs)]
    new[3], new[40] = 90, 40
    _attention(etc, ref.shape(4, 2, 64), kv, new)


@pytest.mark.parametrize("nq,nkv,d", [(16, 8, 64), (9, 3, 128), (10, 5, 64)])
def test_attention_calls_one_after_the_other(etc, nq, nkv, d):
    """Calls of more pieces than workgroups, and of fewer, on one handle: what a workgroup takes next is counted from call to call."""
    s, rng = ref.shape(nq, nkv, d), np.random.default_rng(nq)
    some = lambda n, longest: [int(x) for x in rng.integers(1, longest, n)]      # noqa: E731
    calls = []
    for i, (kv, new) in enumerate((([*some(190, 150)], [1] * 190), (some(3, 200), [1, 2, 40]), ([0, 0, 90, *some(120, 300)], [700, 300, 201] + [1] * 120), ([1500] * 2, [400, 1]))):
        table, n_pages = ref.paged([a + b for a, b in zip(kv, new)], s.page, i)
        (k, ks), (v, vs) = codes.pools(i, n_pages, s.page, nkv, d), codes.pools(i + 9, n_pages, s.page, nkv, d)
        indptr = np.concatenate(([0], np.cumsum(new)))
        q = randn(i, int(indptr[-1]), nq, d)
        want, size = ref.attention(s, q, codes.values(k, ks), codes.values(v, vs), indptr, kv, table)
        calls.append(([q.cuda(), torch.empty(q.shape, dtype=q.dtype, device="cuda"), i32(indptr), i32(kv), i32(table), k.cuda(), v.cuda(), ks.cuda(), vs.cuda()], want, size))
    sv = etc.Serving(s, max_seqs=190, max_tokens=1400, max_kv_len=2000)
    first = {}
    for turn in (0, 1, 2, 3, 0, 0, 2, 2, 1, 3, 2, 0, 3):
        args, want, size = calls[turn]
        args[1].fill_(7.0)
        sv.attention_codes(*args)
        if turn not in first:
            first[turn] = args[1].clone()
            ref.check_attention(args[1], want, size)
        assert torch.equal(args[1], first[turn])
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()


@pytest.mark.parametrize("d", [64, 128])
def test_attention_queries_of_wide_range(etc, d):
    """Elements of a row over many powers of two; rows of zeros; rows so small or so large that their scale is."""
    def change(q):
        q *= torch.exp2(torch.randint(-12, 1, q.shape, generator=torch.Generator().manual_seed(3)).float()).bfloat16()
        q[0] = 0
        q[1] *= 2.0 ** -60
        q[2, 0, 0], q[2, 0, 1:] = 2.0, 0
    for kv, new in (([100], [5]), ([100], [90])):
        _attention(etc, ref.shape(4, 2, d), kv, new, q_change=change)


def _spoil_at(table, page, b, keys, head, code=0x7F, where=0):
    def spoil(k, v, _):
        for t in keys:
            (k, v)[where].view(torch.uint8)[table(_)[b, t // page], t % page, head, 5] = code
    return spoil


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", [0, 1])
@pytest.mark.parametrize("kv,new", [([40, 100], [3, 20]), ([40, 100], [3, 200])])
def test_attention_nan_codes(etc, d, where, kv, new):
    """A NaN among a sequence's last keys reaches the rows that see it, and no others; another sequence none of it."""
    s = ref.shape(4, 2, d)
    at = kv[1] + 7                                       # a new token of sequence 1
    spoil = _spoil_at(lambda t: t, s.page, 1, [at], 1, where=where)

    def check(got, want, size, indptr):
        hit = torch.zeros(got.shape, dtype=torch.bool)
        hit[int(indptr[1]) + 7:int(indptr[2]), 2:, :] = True
        if where == 1:
            hit[..., :5] = False
            hit[..., 6:] = False
        assert torch.equal(torch.isnan(got), hit)
        bound = (2.0 ** -8 * want.abs() + (2.0 ** -12 + 2.0 ** -8) * size + 1e-30)
        assert bool(((got - want).abs() <= bound)[~hit].all())
    _attention(etc, s, kv, new, spoil=spoil, check=check)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_nan_seen_by_all(etc, d):
    s = ref.shape(4, 2, d)
    for new in (2, 100):
        def check(got, want, size, indptr):
            hit = torch.zeros(got.shape, dtype=torch.bool)
            hit[:, :2, 5] = True
            assert torch.equal(torch.isnan(got), hit)
        _attention(etc, s, [90], [new], spoil=_spoil_at(lambda t: t, s.page, 0, [3], 0, code=0xFF, where=1), check=check)


@pytest.mark.parametrize("shift", [-30, 60, 100])
def test_attention_scales(etc, shift):
    """Values from 2^-38 to 2^105: only V's matter there, K's scores stay of ordinary size by q's."""
    for kv, new in (([100, 5], [2, 1]), ([100], [90])):
        _attention(etc, ref.shape(4, 2, 128), kv, new, shift=shift, q_change=lambda q: q.mul_(2.0 ** -shift))


@pytest.mark.parametrize("why", ["page", "page_low", "length", "order", "rows", "table"])
def test_attention_refuses(etc, why):
    s = ref.shape(4, 2, 64)
    kv, new = [100, 40, 64], [2, 70, 1]
    table, n_pages = ref.paged([k + n for k, n in zip(kv, new)], 16, 3)
    (k, ks), (v, vs) = codes.pools(1, n_pages, 16, 2, 64), codes.pools(2, n_pages, 16, 2, 64)
    indptr = np.concatenate(([0], np.cumsum(new)))
    given = {"kv": np.array(kv), "indptr": indptr.copy(), "table": table.copy()}
    if why == "page":
        given["table"][1, 2] = n_pages
    elif why == "page_low":
        given["table"][1, 0] = -1
    elif why == "length":
        given["kv"][1] = -5
    elif why == "order":
        given["indptr"][1], given["indptr"][2] = 72, 2
    elif why == "rows":
        given["indptr"][3] = 1000
    else:
        given["kv"][1] = 16 * table.shape[1]
    q, out = randn(3, 73, 4, 64), torch.zeros(73, 4, 64, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=3, max_tokens=73, max_kv_len=4000)
    dev = [t.cuda() for t in (k, v, ks, vs)]
    sv.attention_codes(q.cuda(), out, i32(given["indptr"]), i32(given["kv"]), i32(given["table"]), *dev)
    code, op, index, value = sv.read_error()
    assert op == 6 and code == (3 if why.startswith("page") else 2)
    want, size = ref.attention(s, q, codes.values(k, ks), codes.values(v, vs), indptr, kv, table)
    for b in {"order": (), "rows": (0, 1)}.get(why, (0, 2)):
        r = slice(int(indptr[b]), int(indptr[b + 1]))
        ref.check_attention(out[r], want[r], size[r])
    sv.attention_codes(q.cuda(), out, i32(indptr), i32(kv), i32(table), *dev)
    assert sv.read_error() == (0, 0, 0, 0)
    ref.check_attention(out, want, size)
    sv.close()


# ---- ends of what is allowed ------------------------------------------------------------------------------------------
def test_append_of_the_most_blocks(etc):
    """2^20 rows of 128 KV heads in pages that workgroups share: more workgroups of K and V than one dimension of a launch takes, the queries'
    behind them.  Nearly all rows are left out."""
    s, rows = ref.shape(128, 128, 64, page=64), 1 << 20
    live = np.concatenate((np.arange(3), np.arange(rows - 70, rows)))
    where = np.concatenate((np.arange(5, 8), np.arange(64 + 60, 64 + 60 + 70)))
    slots = np.full(rows, -1, np.int32)
    slots[live] = where
    x = torch.empty(rows, 128 * 64, dtype=torch.bfloat16, device="cuda")
    q = torch.empty(rows, 128, 64, dtype=torch.bfloat16, device="cuda")
    some = randn(1, len(live), 128 * 64)
    x[torch.as_tensor(live).cuda()] = some.cuda()
    q[3], q[rows - 71] = 7.0, 7.0
    (k0, ks0), (v0, vs0) = codes.pools(2, 4, 64, 128, 64), codes.pools(3, 4, 64, 128, 64)
    k, ks, v, vs = [t.cuda() for t in (k0, ks0, v0, vs0)]
    pos = np.arange(rows) % 5000
    sv = etc.Serving(s, max_seqs=1, max_tokens=rows, max_kv_len=100)
    sv.append_codes(x, x, x, i32(pos), i32(slots), q, k, v, ks, vs)
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    heads = some.view(-1, 128, 64)
    want, size = ref.rotate(s, heads, pos[live])
    got = q[torch.as_tensor(live).cuda()].cpu().double()
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + FP32 * size).all())
    assert bool((q[3] == 7.0).all()) and bool((q[rows - 71] == 7.0).all())
    codes.check_append(64, where, want, FP32 * size, k0, ks0, k, ks)
    codes.check_append(64, where, heads.double(), torch.zeros(heads.shape, dtype=torch.float64), v0, vs0, v, vs)
    del x, q
    torch.cuda.empty_cache()                             # 34 GB that no other test asks for


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_seqs,new,keys", [(40, 1, 4096), (40, 20, 2048), (20, 129, 4096)])
@pytest.mark.parametrize("top", [False, True])
def test_attention_ends_of_scales(etc, d, n_seqs, new, keys, top):
    """The least scale and, for so many keys, the largest.  The first keys, 32 of every wavefront, score nearly 2^8 below the
    others, so that those have weights near 2^8, the most that a reference that lags lets through; the largest case has values of 384 to 448 of one sign in every column.
    Sequences share their pages, and there are enough of them that none is cut."""
    s, page = ref.shape(16, 8, d), 16
    n_pages = keys // page
    v_byte = 238 - int(math.log2(keys)) if top else 27
    k_byte = 227 if top else 27
    table, _ = ref.paged([keys], page, 3, extra=0)
    k0 = torch.zeros(n_pages, page, 8, d)
    k0[torch.as_tensor(table[0, 256 // page:n_pages]).long(), :, :, 0] = 44.0 if d == 64 else 60.0      # times 1 / ln 2 / sqrt(d): 7.93, 7.65
    g = torch.Generator().manual_seed(d)
    v0 = (384 + 32 * torch.randint(0, 3, (n_pages, page, 8, d), generator=g)) * (torch.randint(0, 2, (8, d), generator=g) * 2 - 1) if top else \
        torch.randn(n_pages, page, 8, d, generator=g) * 100
    k, v = k0.to(torch.float8_e4m3fn), v0.float().clamp(-448, 448).to(torch.float8_e4m3fn)
    ks, vs = [torch.full((n_pages, 8), b, dtype=torch.uint8) for b in (k_byte, v_byte)]
    q = torch.zeros(new, 16, d)
    q[..., 0] = 2.0 ** (127 - k_byte)
    rows = n_seqs * new
    out = torch.zeros(rows, 16, d, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=n_seqs, max_tokens=rows, max_kv_len=keys)
    sv.attention_codes(q.bfloat16().repeat(n_seqs, 1, 1).cuda(), out, i32(new * np.arange(n_seqs + 1)), i32([keys - new] * n_seqs), i32(np.repeat(table, n_seqs, 0)),
                       k.cuda(), v.cuda(), ks.cuda(), vs.cuda())
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    want, size = ref.attention(s, q.bfloat16(), codes.values(k, ks), codes.values(v, vs), [0, new], [keys - new], table)
    got = out.cpu().double().view(n_seqs, new, 16, d)
    # as _attention's; and what is below 2^-126 of a probability times a scale, or of a product, is lost: at most 448 * 2^-126 of a key, twice
    few = new * 2 <= 64
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -12 + (0 if few else 2.0 ** -8)) * size + keys * 2.0 ** -116
    worst = float(((got - want).abs() / bound).max())
    assert worst <= 1.0, f"worst error / bound {worst:.3f}"


@pytest.mark.parametrize("page", [1, 2, 4])
@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (6, 2, 128), (8, 1, 128)])
def test_attention_pairs_with_windows(etc, page, nq, nkv, d):
    """Blocks of 33 to 64 rows, whose wavefronts share a ring, over more pages than a window of their ids holds; NaN codes among what no row sees."""
    rows = 64 // (nq // nkv)
    _attention(etc, ref.shape(nq, nkv, d, page=page), [600 - rows], [rows])                  # one piece, three windows of single tokens
    _attention(etc, ref.shape(nq, nkv, d, page=page), [5000, 255, 590, 9000], [rows, rows // 2 + 1, rows - 1, rows], seed=7)


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (6, 2, 128)])
def test_attention_pairs_with_windows_not_cut(etc, nq, nkv, d):
    """The same in pieces of several thousand keys."""
    rows = 64 // (nq // nkv)
    _attention(etc, ref.shape(nq, nkv, d, page=2), [1500 + 7 * b for b in range(150)], [rows - b % 3 for b in range(150)])
