"""The cache of codes as a server uses it: tables, append, attention and scores together, eager, captured, on several streams."""
import numpy as np
import pytest
import torch

import codes_ref as codes
import serving_ref as ref
from serving_ref import i32

pytestmark = pytest.mark.gpu

FP32 = 2.0 ** -19                                        # tests/test_gpu_codes.py


@pytest.fixture(scope="module")
def etc():
    import paper_2604_13327_amd
    return paper_2604_13327_amd


def _zero(*size, dtype=torch.int32):
    return torch.zeros(*size, dtype=torch.uint8, device="cuda").to(dtype)


class State:
    """A server's arrays, on the GPU: one layer's cache of codes, tables, rows of a step."""

    def __init__(self, s, seqs, rows, n_pages, top):
        self.s, self.seqs, self.rows = s, seqs, rows
        self.table, self.count, self.count_after = _zero(seqs, n_pages), i32([n_pages]), i32([0])
        self.free = torch.arange(n_pages, dtype=torch.int32, device="cuda").flip(0).contiguous()
        self.q_indptr, self.slots, self.positions, self.status, self.kv_after = _zero(seqs + 1), _zero(rows), _zero(rows), _zero(1), _zero(seqs)
        self.q, self.out = (_zero(rows, s.nq, s.d, dtype=torch.bfloat16) for _ in range(2))
        self.k, self.v = (_zero(n_pages, s.page, s.nkv, s.d, dtype=torch.float8_e4m3fn) for _ in range(2))
        self.ks, self.vs = (_zero(n_pages, s.nkv, dtype=torch.uint8).view(torch.float8_e8m0fnu) for _ in range(2))
        self.logprob, self.entropy = (_zero(rows, dtype=torch.float32) for _ in range(2))
        self.ids, self.tops = _zero(rows, top), _zero(rows, top, dtype=torch.float32)

    def step(self, sv, kv, new, qkv, gq, gk, logits, tokens):
        s, a, b = self.s, self.s.nq * self.s.d, (self.s.nq + self.s.nkv) * self.s.d
        sv.tables(kv, new, self.table, self.free, self.count, q_indptr=self.q_indptr, slots=self.slots, positions=self.positions,
                  status=self.status, free_count_out=self.count_after, total_len=self.kv_after)
        sv.append_codes(qkv[:, :a], qkv[:, a:b], qkv[:, b:], self.positions, self.slots, self.q, self.k, self.v, self.ks, self.vs, gq=gq, gk=gk)
        sv.attention_codes(self.q, self.out, self.q_indptr, kv, self.table, self.k, self.v, self.ks, self.vs)
        sv.score(logits, tokens, self.logprob, self.entropy, self.ids, self.tops)

    def outputs(self):
        return {n: t.view(torch.uint8) if t.dtype in (torch.float8_e4m3fn, torch.float8_e8m0fnu) else t for n, t in vars(self).items() if isinstance(t, torch.Tensor)}


def test_steps(etc):
    """Chunks and single tokens that grow, so that scales of pages begun do: every step's pools against the exact append to the pools before
    it, its attention against the exact one over the pools it left."""
    s, seqs, rows = ref.shape(4, 2, 64, qk_norm=True, vocab=300, theta=1e5), 4, 160
    t, sv = State(s, seqs, rows, 60, 3), etc.Serving(s, max_seqs=seqs, max_tokens=rows, max_kv_len=400)
    g = torch.Generator().manual_seed(1)
    gq, gk = (1 + 0.3 * torch.randn(2, s.d, generator=g)).bfloat16()
    kv, grown = [0] * seqs, 0
    for i, new in enumerate(([20, 3, 0, 100], [1, 1, 5, 1], [1, 1, 1, 1], [1, 0, 1, 1], [40, 17, 1, 90], [1, 1, 1, 1], [1, 1, 1, 1], [0, 1, 1, 0])):
        qkv = (torch.randn(rows, 512, generator=g) * 1.7 ** i).bfloat16()
        logits, tokens = torch.randn(rows, 300, generator=g), np.where(np.arange(rows) < sum(new), i, -1)
        before = [x.cpu() for x in (t.k, t.ks, t.v, t.vs)]
        t.step(sv, i32(kv), i32(new), qkv.cuda(), gq.cuda(), gk.cuda(), logits.cuda(), i32(tokens))
        assert sv.read_error() == (0, 0, 0, 0) and int(t.status) == 0
        n, slots, heads = sum(new), t.slots.cpu().numpy(), qkv.view(rows, 8, 64)
        want, size = ref.rotate(s, heads[:, 4:6], t.positions.cpu(), gk)
        codes.check_append(s.page, slots, want, FP32 * size, before[0], before[1], t.k, t.ks)
        vv = heads[:, 6:].double()
        codes.check_append(s.page, slots, vv, torch.zeros_like(vv), before[2], before[3], t.v, t.vs)
        grown += int((t.vs.cpu().view(torch.uint8) > before[3].view(torch.uint8)).sum())
        out, size = ref.attention(s, t.q, codes.values(t.k, t.ks), codes.values(t.v, t.vs), t.q_indptr.tolist(), kv, t.table.cpu().numpy())
        ref.check_attention(t.out[:n], out[:n], size[:n])
        for r in range(0, n, 7):
            lp, entropy, ids, tops = codes.score(logits[r].numpy(), i, 3)
            assert abs(float(t.logprob[r]) - lp) < 2e-5 and abs(float(t.entropy[r]) - entropy) < 1e-4 and t.ids[r].tolist() == ids.tolist()
        assert not t.logprob[n:].any() or i
        kv = [a + b for a, b in zip(kv, new)]
        t.count.copy_(t.count_after)
    assert grown > 40
    sv.close()


def test_captured_step_follows_its_arrays(etc):
    """The four calls in one graph: replayed with other lengths, tables and inputs, with eager work of a second handle and synchronizations in
    between, every replay equal to the eager calls."""
    s, seqs, rows = ref.shape(8, 2, 128, qk_norm=True, vocab=20000), 4, 600
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *size, dtype=torch.bfloat16: torch.randn(*size, device="cuda", generator=g).to(dtype)        # noqa: E731
    svs = [etc.Serving(s, max_seqs=seqs, max_tokens=rows, max_kv_len=2000) for _ in range(2)]
    gq, gk, qkv, logits, tokens = 1 + rnd(128), 1 + rnd(128), rnd(rows, 12 * 128), rnd(9, 20000), i32([5, 7, -1, 9, 0, 19999, 3, 3, 4])
    kv, new, states = i32([0] * 4), i32([1] * 4), [State(s, seqs, rows, 400, 20) for _ in range(2)]
    for t in states:                                     # nine rows of logits, as their own arrays
        t.logprob, t.entropy, t.ids, t.tops = t.logprob[:9].clone(), t.entropy[:9].clone(), t.ids[:9].clone(), t.tops[:9].clone()
    args = (kv, new, qkv, gq, gk, logits, tokens)
    for sv, t in zip(svs, states):
        t.step(sv, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        states[0].step(svs[0], *args)
    for lens in ([3, 500, 0, 60], [1, 1, 1, 1], [0, 0, 0, 0], [256, 7, 30, 300], [2, 90, 100, 3], [1, 1, 1, 1]):
        new.copy_(i32(lens))
        qkv.copy_(rnd(rows, 12 * 128))
        logits.copy_(rnd(9, 20000))
        graph.replay()
        states[1].step(svs[1], *args)
        torch.cuda.synchronize()
        a, b = states[0].outputs(), states[1].outputs()
        for name in a:
            assert torch.equal(a[name], b[name]), (name, lens)
        assert int(states[0].status) == 0
        kv.copy_(states[0].kv_after)
        for t in states:
            t.count.copy_(t.count_after)
        rnd(1 << 20).sum().item()
    for sv in svs:
        assert sv.read_error()[0] == 0
        sv.close()


def test_two_graphs_of_one_handle(etc):
    """Captured calls of different sizes share the handle's workspace: replayed in turn on one stream."""
    s = ref.shape(8, 2, 128, vocab=40000)
    sv = etc.Serving(s, max_seqs=3, max_tokens=300, max_kv_len=6400)
    (k, ks), (v, vs) = (tuple(x.cuda() for x in codes.pools(i, 1200, 16, 2, 128)) for i in (1, 2))
    table = i32(np.random.default_rng(1).permutation(1200).reshape(3, 400))
    calls = []
    for new, kv, rows in (([1, 1, 1], [6000, 100, 4000], 3), ([200, 1, 99], [5000, 6300, 0], 40)):
        q = ref.randn(sum(new), sum(new), 8, 128).cuda()
        logits = ref.randn(rows, rows, 40000).cuda()
        out = {"o": torch.zeros_like(q), "lp": _zero(rows, dtype=torch.float32), "ids": _zero(rows, 20)}
        given = (q, i32(np.concatenate(([0], np.cumsum(new)))), i32(kv), logits, i32(np.arange(rows)))

        def call(given=given, out=out):
            q, indptr, kv, logits, tokens = given
            sv.attention_codes(q, out["o"], indptr, kv, table, k, v, ks, vs)
            sv.score(logits, tokens, out["lp"], top_ids=out["ids"])
        call()
        torch.cuda.synchronize()
        want = {n: x.clone() for n, x in out.items()}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        calls.append((graph, out, want, given))          # its inputs live as long as the graph
    for _ in range(4):
        for graph, out, *_ in calls:
            for x in out.values():
                x.zero_()
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for _, out, want, _ in calls for n in out)
    assert sv.read_error() == (0, 0, 0, 0)
    sv.close()


def test_handles_on_streams_of_their_own(etc):
    """Two handles on two streams, without waiting for each other; a call goes to the stream it is given."""
    s = ref.shape(8, 2, 128, vocab=30000)
    (k, ks), (v, vs) = (tuple(x.cuda() for x in codes.pools(i, 400, 16, 2, 128)) for i in (1, 2))
    q, qi, kv = ref.randn(1, 70, 8, 128).cuda(), i32([0, 1, 70]), i32([3000, 3000])
    table, logits, tokens = i32(np.random.default_rng(1).permutation(400).reshape(2, 200)), ref.randn(4, 5, 30000).cuda(), i32([0, 1, 2, 3, 4])
    svs, streams = [etc.Serving(s, max_seqs=2, max_tokens=70, max_kv_len=3200) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    make = lambda: (torch.zeros_like(q), _zero(5, dtype=torch.float32), _zero(5, 9))      # noqa: E731
    want, got = make(), [[make() for _ in svs] for _ in range(6)]
    call = lambda sv, o, st: (sv.attention_codes(q, o[0], qi, kv, table, k, v, ks, vs, stream=st), sv.score(logits, tokens, o[1], top_ids=o[2], stream=st))      # noqa: E731
    call(svs[0], want, None)
    torch.cuda.synchronize()
    for pair in got:
        for sv, o, st in zip(svs, pair, streams):
            call(sv, o, st)
    for st in streams:
        st.synchronize()
    assert all(torch.equal(a, b) for pair in got for o in pair for a, b in zip(o, want))
    for sv in svs:
        assert sv.read_error()[0] == 0
        sv.close()
