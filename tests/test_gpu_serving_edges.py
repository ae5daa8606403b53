"""Serving operators on the GPU where a value or an id is none that a kernel can go on with: infinities and NaN among the values a
row sees, page ids of no pool."""
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


# ---- attention: what is no number arrives as what it is ----------------------------------------------------------------
def _same_kinds(got, want):
    """+inf, -inf and NaN each where the 64-bit form has them."""
    got = got.double().cpu()
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got), kind(want)), f"{kind.__name__}: {int(kind(got).sum())} of {int(kind(want).sum())}"


def _attend_to(etc, s, kv, new, odd, seed=0):
    """`odd`: (sequence, position, first element, value): V there and at every 7th element behind it."""
    table, n_pages = ref.paged([a + b for a, b in zip(kv, new)], s.page, seed)
    q_indptr = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
    q, k, v = (randn(seed + i, *size) for i, size in ((1, (int(q_indptr[-1]), s.nq, s.d)), (2, (n_pages, s.page, s.nkv, s.d)),
                                                     (3, (n_pages, s.page, s.nkv, s.d))))
    for b, pos, e, value in odd:
        v[int(table[b, pos // s.page]), pos % s.page, :, e::7] = value
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=len(kv), max_tokens=int(q_indptr[-1]), max_kv_len=max(a + b for a, b in zip(kv, new)))
    sv.attention(q.cuda(), out, i32(q_indptr), i32(kv), i32(table), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()
    want, size = ref.attention(s, q, k, v, q_indptr, kv, table)
    _same_kinds(out, want)
    ref.check_attention(out, want, size)


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 128), (4, 2, 64), (8, 8, 64)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("kv,new,pos", [([0], [1], 0), ([0], [9], 3), ([0], [130], 3), ([40], [2], 40), ([40], [100], 41), ([127], [1], 127),
                                        ([128], [1], 128), ([64], [70], 70), ([5000], [3], 5001), ([5000], [90], 5030), ([5000], [90], 17), ([5000], [3], 17)])
def test_attention_infinities_a_row_sees(etc, nq, nkv, d, value, kv, new, pos):
    """In tiles seen whole, in tiles some rows see a part of, and in the first tile of a row or of a piece of its keys."""
    _attend_to(etc, ref.shape(nq, nkv, d), kv, new, [(0, pos, 2, value)])


@pytest.mark.parametrize("kv,new", [([0], [60]), ([0], [8]), ([30], [30]), ([200, 0], [100, 60])])
def test_attention_infinities_of_both_signs(etc, kv, new):
    """+inf in one element, -inf in another; where both meet in one, NaN from the later token on."""
    a, b = kv[0] + 1, kv[0] + new[0] // 2
    _attend_to(etc, ref.shape(8, 2, 128), kv, new, [(0, a, 0, math.inf), (0, a, 1, -math.inf), (0, b, 1, math.inf), (0, b, 3, -math.inf), (0, b + 2, 4, math.nan)])


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("kv,new", [([300], [1]), ([2000, 10], [5, 1]), ([900], [70])])
def test_attention_infinities_of_every_key(etc, nq, nkv, d, kv, new):
    """Every probability times an infinity, those of a single bf16 part among them (the largest score's is 1)."""
    every = [(b, pos, e, value) for b in range(len(kv)) for pos in range(kv[b] + new[b]) for e, value in ((0, math.inf), (1, -math.inf))]
    _attend_to(etc, ref.shape(nq, nkv, d), kv, new, every)


@pytest.mark.parametrize("gap", [20.0, 45.0, 65.0])
@pytest.mark.parametrize("new", [1, 3, 90])
def test_attention_infinities_of_small_probability(etc, gap, new):
    """Probabilities down to e^-65 (2^-94), in a tile seen whole and in the last one; what a row does not see leaves no trace."""
    s, kv = ref.shape(4, 2, 64), 300
    table, n_pages = ref.paged([kv + new], 16, 1)
    q, k, v = torch.zeros(new, 4, 64), torch.zeros(n_pages, 16, 2, 64), randn(2, n_pages, 16, 2, 64)
    q[:, :, 0], q[:, :, 1] = gap / 2, 1.0
    at = lambda pos: (int(table[0, pos // 16]), pos % 16)        # noqa: E731
    k[at(7)][:, 0] = 16.0                                 # scores 0 but for this one's, q . k / sqrt(64) = gap
    k[..., 1] = (randn(3, n_pages, 16, 2) * 4).float()    # and the others' about 0, so that probabilities are of all kinds
    for pos, e, value in ((40, 0, math.inf), (90, 1, -math.inf), (kv, 2, math.inf), (kv + new - 1, 3, -math.inf), (120, 4, 3.3e38), (kv + new - 1, 5, -3.3e38)):
        v[at(pos)][:, e] = value
    q, k = q.bfloat16(), k.bfloat16()
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=1, max_tokens=new, max_kv_len=kv + new)
    sv.attention(q.cuda(), out, i32([0, new]), i32([kv]), i32(table), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    sv.close()
    want, size = ref.attention(s, q, k, v, [0, new], [kv], table)
    _same_kinds(out, want)
    ref.check_attention(out[..., :4], want[..., :4], size[..., :4])
    ref.check_attention(out[..., 6:], want[..., 6:], size[..., 6:])


def _cancelling(etc, s, kv, new, seed):
    """Values of both signs that nearly cancel: (what came out, the 64-bit form, the sum of p |v|)."""
    table, n_pages = ref.paged([a + b for a, b in zip(kv, new)], s.page, seed)
    q_indptr = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
    q, k, v = randn(seed, int(q_indptr[-1]), s.nq, s.d), randn(seed + 1, n_pages, s.page, s.nkv, s.d), randn(seed + 2, n_pages, s.page, s.nkv, s.d)
    v = (1000.0 * v.sign() + v.float()).bfloat16()
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    sv = etc.Serving(s, max_seqs=len(kv), max_tokens=int(q_indptr[-1]), max_kv_len=max(a + b for a, b in zip(kv, new)))
    sv.attention(q.cuda(), out, i32(q_indptr), i32(kv), i32(table), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    sv.close()
    want, size = ref.attention(s, q, k, v, q_indptr, kv, table)
    return out.double().cpu(), want, size


# Rounding of the result (2^-8 of it), and of scores, exponentials and sums (2^-12 of the sum of p |v|, tests/serving_ref.py)
@pytest.mark.parametrize("nq,nkv,d,kv,new", [(8, 2, 128, [1], [1]), (8, 2, 128, [300, 40], [5, 1]), (4, 2, 64, [700], [32]), (64, 8, 128, [6000, 90], [1, 8])])
def test_attention_of_few_rows_keeps_its_probabilities(etc, nq, nkv, d, kv, new):
    """At most 64 rows (tokens times heads to a KV head): a probability is two bf16 parts, exact to 2^-15 (the upper part leaves less than
    2^-7 of it, the rest is rounded by 2^-8 of that)."""
    got, want, size = _cancelling(etc, ref.shape(nq, nkv, d), kv, new, 11)
    err, bound = (got - want).abs(), 2.0 ** -8 * want.abs() + (2.0 ** -12 + 2.0 ** -15) * size
    assert bool((err <= bound).all()), f"worst error / bound {float((err / bound).max()):.3f}"


@pytest.mark.parametrize("nq,nkv,d,kv,new", [(8, 2, 128, [300, 0], [17, 100]), (4, 2, 64, [700], [33]), (64, 8, 128, [6000, 90], [9, 40])])
def test_attention_of_many_rows_rounds_its_probabilities(etc, nq, nkv, d, kv, new):
    """More: half a unit of bf16 each, 2^-8 of the sum of p |v| at most, whatever cancels; and again in the sum they are divided by."""
    got, want, size = _cancelling(etc, ref.shape(nq, nkv, d), kv, new, 12)
    err, bound = (got - want).abs(), 2.0 ** -8 * (2 * want.abs() + size) + 2.0 ** -12 * size
    assert bool((err <= bound).all()), f"worst error / bound {float((err / bound).max()):.3f}"


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (64, 8, 128), (8, 8, 128)])
@pytest.mark.parametrize("kv,new", [([0], [1]), ([383], [1]), ([384], [1]), ([5000], [1]), ([900], [60]), ([2000, 1500, 10], [1, 3, 1]), ([700] * 40, [1] * 40)])
def test_attention_of_a_handle_with_tight_limits(etc, nq, nkv, d, kv, new):
    """The workspace follows the limits; the way keys are cut, and so every bit, is that of a handle with room for everything."""
    s = ref.shape(nq, nkv, d)
    total = [a + b for a, b in zip(kv, new)]
    table, n_pages = ref.paged(total, 16, 3)
    q, k, v = randn(1, sum(new), nq, d).cuda(), randn(2, n_pages, 16, nkv, d).cuda(), randn(3, n_pages, 16, nkv, d).cuda()
    outs = []
    for limits in ((len(kv), sum(new), max(total)), (1024, 1 << 16, 1 << 20)):
        sv = etc.Serving(s, *limits)
        out = torch.zeros_like(q)
        for _ in range(2):
            sv.attention(q, out, i32(np.concatenate(([0], np.cumsum(new)))), i32(kv), i32(table), k, v)
        assert sv.read_error() == (0, 0, 0, 0)
        sv.close()
        outs.append(out)
    assert torch.equal(*outs)


# ---- tables: page ids of no pool --------------------------------------------------------------------------------------
PAGE, N_PAGES, KV, NEW = 16, 8, [20, 5, 0], [3, 30, 18]


@pytest.mark.parametrize("where", ["table", "free"])
@pytest.mark.parametrize("bad", [-1, -(1 << 31), 1 << 27, 1 << 28, (1 << 28) + 1, 1 << 30, (1 << 31) - 1])
def test_tables_hand_on_no_slot_of_a_page_id_out_of_range(etc, where, bad):
    """An id below 0 or of more tokens than 31 bits count: `id * page` in 32 bits is a slot of another page, or a negative one that
    stands for padding.  Its tokens get a slot that append refuses, and tables reports it; everything else is as ever."""
    s = ref.shape(4, 2, 64, page=PAGE)
    sv = etc.Serving(s, max_seqs=3, max_tokens=60, max_kv_len=64)
    table, free = np.full((3, 4), -7, np.int32), [7, 6, 5, 4, 3]      # taken from the end: 3, 4 (sequence 1), 5, 6 (2)
    table[0, :2], table[1, 0] = [0, 1], 2
    if where == "table":
        table[0, 1], seq = bad, 0                         # positions 20 .. 22 lie in it
    else:
        free[3], seq = bad, 1                             # the second page of sequence 1's two, positions 32 .. 34
    rows = 55                                             # 51 tokens and padding
    e = lambda n: torch.full((n,), 12345, dtype=torch.int32, device="cuda")        # noqa: E731
    o = {"q_indptr": e(4), "slots": e(rows), "positions": e(rows), "status": e(1), "total_len": e(3)}
    t, count = i32(table), i32([len(free)])
    sv.tables(i32(KV), i32(NEW), t, i32(free), count, **o)
    assert sv.read_error() == (3, 1, seq, bad)
    want = ref.tables(KV, NEW, table, free, PAGE, rows)
    slots = np.array([x if 0 <= x < 1 << 31 else (1 << 31) - 1 for x in want["slots"][:51]] + [-1] * 4)
    held = {"table": slice(0, 3), "free": slice(3 + 27, 3 + 30)}[where]      # the rows of the bad page's tokens
    slots[held] = (1 << 31) - 1
    assert np.array_equal(o["slots"].cpu().numpy(), slots)
    for name in ("q_indptr", "positions", "status", "total_len"):
        assert np.array_equal(o[name].cpu().numpy(), np.asarray(want[name])), name
    assert np.array_equal(t.cpu().numpy(), want["block_table"]) and int(count) == 1

    pools = [randn(i, N_PAGES, PAGE, 2, 64).cuda() for i in (1, 2)]
    before = [p.clone() for p in pools]
    q, k, v, out = randn(3, rows, 256).cuda(), randn(4, rows, 128).cuda(), randn(5, rows, 128).cuda(), torch.full((rows, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    sv.append(q, k, v, o["positions"], o["slots"], out, *pools)
    word = sv.read_error()
    assert word[:2] == (1, 2) and held.start <= word[2] < held.stop and word[3] == (1 << 31) - 1
    written = torch.zeros(N_PAGES * PAGE, dtype=torch.bool)
    written[[int(x) for x in slots if 0 <= x < N_PAGES * PAGE]] = True
    for p, b in zip(pools, before):
        same = (p == b).view(N_PAGES * PAGE, -1).all(1).cpu()
        assert torch.equal(same, ~written)
    good = [r for r, x in enumerate(slots) if 0 <= x < N_PAGES * PAGE]
    assert torch.equal(pools[1].view(-1, 128)[torch.as_tensor(slots[good]).cuda()], v[good])
    assert bool((out[held] == 7.0).all()) and sv.read_error() == (0, 0, 0, 0)
    sv.close()


def test_tables_page_ids_to_the_end_of_their_range(etc):
    """Pages of one token and of 16: the last id whose slots fit 31 bits."""
    for page, last in ((1, (1 << 31) - 2), (16, (1 << 27) - 1)):
        sv = etc.Serving(ref.shape(page=page), max_seqs=1, max_tokens=1, max_kv_len=16)
        o = {n: i32([5] * k) for n, k in (("q_indptr", 2), ("slots", 1), ("positions", 1), ("status", 1))}
        sv.tables(i32([0]), i32([1]), i32([[0]]), i32([last]), i32([1]), **o)
        assert int(o["slots"]) == last * page and int(o["status"]) == 0 and sv.read_error() == (0, 0, 0, 0)
        sv.close()


# ---- reports ----------------------------------------------------------------------------------------------------------
def test_a_report_is_of_one_refusal(etc):
    """Many rows refused at once, by many wavefronts: index and value belong together."""
    s, n = ref.shape(4, 2, 64), 8192
    sv = etc.Serving(s, max_seqs=1, max_tokens=n, max_kv_len=100)
    q, k, v = (torch.zeros(n, w, dtype=torch.bfloat16, device="cuda") for w in (256, 128, 128))
    out, pools = torch.zeros(n, 4, 64, dtype=torch.bfloat16, device="cuda"), [torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    positions = i32(np.zeros(n))
    for trial in range(20):
        base = 1000 + 10000 * trial
        sv.append(q, k, v, positions, i32(base + np.arange(n)), out, *pools)
        word = sv.read_error()
        assert word[:2] == (1, 2) and word[3] == base + word[2], word
    sv.close()
