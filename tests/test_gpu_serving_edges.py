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
                                        ([128], [1], 128), ([64], [70], 70), ([5000], [3], 5001), ([5000], [90], 5030), ([5000], [90], 17)])
def test_attention_infinities_a_row_sees(etc, nq, nkv, d, value, kv, new, pos):
    """In tiles seen whole, in tiles some rows see a part of, and in the first tile of a row or of a piece of its keys."""
    _attend_to(etc, ref.shape(nq, nkv, d), kv, new, [(0, pos, 2, value)])


@pytest.mark.parametrize("kv,new", [([0], [60]), ([0], [8]), ([30], [30]), ([200, 0], [100, 60])])
def test_attention_infinities_of_both_signs(etc, kv, new):
    """+inf in one element, -inf in another; where both meet in one, NaN from the later token on."""
    a, b = kv[0] + 1, kv[0] + new[0] // 2
    _attend_to(etc, ref.shape(8, 2, 128), kv, new, [(0, a, 0, math.inf), (0, a, 1, -math.inf), (0, b, 1, math.inf), (0, b, 3, -math.inf), (0, b + 2, 4, math.nan)])
