"""The serving operators together, as a server uses them: a prompt in ragged chunks through a whole (tiny) decoder into the paged
cache, then decode steps of the megakernel on that cache with sampled tokens; and the same calls captured into graphs."""
import dataclasses

import numpy as np
import pytest
import torch

import serving_ref as ref
from serving_ref import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def etc():
    import paper_2604_13327_amd
    return paper_2604_13327_amd


class Pages:
    """A server's page state on the GPU."""

    def __init__(self, n_seqs, cols, n_pages, seed):
        rng = np.random.default_rng(seed)
        self.table = torch.zeros(n_seqs, cols, dtype=torch.int32, device="cuda")
        self.free, self.count = i32(rng.permutation(n_pages)), i32([n_pages])
        self.kv = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")

    def grow(self, sv, new, rows):
        e = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")        # noqa: E731
        n = self.kv.shape[0]
        before = self.kv.clone()
        o = {"q_indptr": e(n + 1), "slots": e(rows), "positions": e(rows), "status": e(1), "page_indptr": e(n + 1), "page_ids": e(self.free.shape[0])}
        sv.tables(self.kv, new, self.table, self.free, self.count, total_len=self.kv, **o)
        return before, o


def _norm(x, g, eps):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * g.float()


def _chunk_forward(s, sv, m, x, kv, o, pools):
    """One chunk through all layers: projections by torch, everything that touches the cache by the serving operators."""
    for layer, w in enumerate(m.weights):
        mm = lambda t, n: t @ w[n].float().t()        # noqa: B023, E731
        h = _norm(x, w["g1"], s.eps)
        q, k, v = (mm(h, n) for n in ("wq", "wk", "wv"))
        q_out = torch.zeros(x.shape[0], s.nq, s.d, dtype=torch.bfloat16, device="cuda")
        out = torch.zeros_like(q_out)
        sv.append(q, k, v, o["positions"], o["slots"], q_out, pools[0][layer], pools[1][layer], gq=w.get("gq"), gk=w.get("gk"))
        sv.attention(q_out, out, o["q_indptr"], kv, o["table"], pools[0][layer], pools[1][layer])
        x = x + mm(out.reshape(x.shape[0], -1).float(), "wo")
        h = _norm(x, w["g2"], s.eps)
        x = x + mm(torch.nn.functional.silu(mm(h, "wg")) * mm(h, "wu"), "wd")
    return x


def test_prompt_in_chunks_then_decode_with_sampling(etc):
    import synth
    from harness import GpuModel
    from synth import gpu as sgpu
    s = synth.TINY_LM
    n_pages, B, lens = 64, 3, [37, 5, 90]
    m = GpuModel(s, seed=3, n_pool_pages=n_pages)
    lm = sgpu.lm_weights_gpu(s, 3, "cuda")
    rng = np.random.default_rng(4)
    prompts = [rng.integers(0, s.vocab, n) for n in lens]
    sv = etc.Serving(s, max_seqs=B, max_tokens=128, max_kv_len=128)

    # the prompts, in chunks: ragged, one sequence idle in one of them, a padded batch
    pools = (torch.full_like(m.kpool, float("nan")), torch.full_like(m.vpool, float("nan")))
    pages, at, last = Pages(B, 8, n_pages, 1), [0] * B, [None] * B
    for step in ([20, 5, 64], [17, 0, 25], [0, 0, 1]):
        new = i32(step)
        before, o = pages.grow(sv, new, 100)
        o["table"] = pages.table
        tokens = np.concatenate([prompts[b][at[b]:at[b] + n] for b, n in enumerate(step)] + [np.zeros(100 - sum(step), np.int64)])
        x = lm["embed"][torch.as_tensor(tokens).cuda()].float()
        x = _chunk_forward(s, sv, m, x, before, o, pools)
        assert int(o["status"]) == 0
        row = 0
        for b, n in enumerate(step):
            row += n
            at[b] += n
            if n:
                last[b] = x[row - 1]
    assert at == lens and pages.kv.tolist() == lens
    logits = _norm(torch.stack(last), lm["gf"], s.eps) @ lm["wlm"].float().t()

    # the same prompts token by token through the megakernel, on a cache of its own with the same pages
    dec = etc.Decoder(s, kv_chunk_tokens=16, sampled_batches=[1, B], max_kv_len=128)
    kp, vp = torch.zeros_like(m.kpool), torch.zeros_like(m.vpool)
    for layer, w in enumerate(m.weights):
        dec.bind_layer_weights(layer, w)
    dec.bind_kv_pool(kp, vp)
    dec.bind_lm_head(lm["embed"], lm["gf"], lm["wlm"])
    want, tok, table = torch.empty(B, s.vocab, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda"), pages.table.cpu().numpy()
    for b in range(B):
        for t in range(lens[b]):
            n = ref.pages_needed(t + 1, s.page)
            dec.bind_step(synth.Step(1, np.array([t], np.int32), np.array([0, n], np.int32), table[b, :n].copy()))
            dec.launch_tokens(tok, token_in=i32([prompts[b][t]]), logits_out=want[b:b + 1])
    torch.cuda.synchronize()
    # both paths round keys, values and attention outputs to bf16 (the decoder keeps the step's own row unrounded): two layers of
    # 2^-8 relative each, against the framework's bar of 2e-2 of the RMS
    rms = want.pow(2).mean().sqrt()
    assert float((logits - want).abs().max() / rms) < 2e-2
    for b in range(B):
        for mine, theirs in zip(pools, (kp, vp)):
            t = torch.arange(lens[b])
            at_ = (torch.as_tensor(table[b].astype(np.int64))[t // s.page].cuda(), (t % s.page).cuda())
            for layer in range(s.n_layers):
                a, c = mine[layer][at_].float(), theirs[layer][at_].float()
                assert float((a - c).abs().max() / c.pow(2).mean().sqrt()) < 2e-2

    # decode steps on the cache the chunks filled, every sequence with its own settings; pages grown on the GPU
    dec2 = etc.Decoder(s, kv_chunk_tokens=16, sampled_batches=[B], max_kv_len=128)
    for layer, w in enumerate(m.weights):
        dec2.bind_layer_weights(layer, w)
    dec2.bind_kv_pool(*pools)
    dec2.bind_lm_head(lm["embed"], lm["gf"], lm["wlm"])
    setting = dict(temperature=torch.tensor([0.0, 0.8, 1.2], device="cuda"), top_k=i32([0, 40, 0]), top_p=torch.tensor([1.0, 0.9, 0.95], device="cuda"))
    token, scratch, out = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    u = torch.rand(6, B, generator=torch.Generator().manual_seed(1))
    sv.sample(logits, u[0].cuda(), token, **setting)
    lg = torch.empty(B, s.vocab, device="cuda")
    for step in range(5):
        kv = pages.kv.cpu().numpy()
        _, o = pages.grow(sv, i32([1] * B), B)
        indptr = o["page_indptr"].cpu().numpy()
        dec2.bind_step(synth.Step(B, kv, indptr, o["page_ids"].cpu().numpy()[:indptr[-1]]))
        dec2.launch_tokens(scratch, token_in=token, logits_out=lg)
        sv.sample(lg, u[step + 1].cuda(), out, **setting)
        torch.cuda.synchronize()
        host = lg.double().cpu().numpy()
        for b in range(B):
            t, _, _, gap = ref.sample_row(host[b], float(u[step + 1, b]), float(np.float32(setting["temperature"][b].item())),
                                          int(setting["top_k"][b]), float(np.float32(setting["top_p"][b].item())))
            assert gap < 1e-7 or int(out[b]) == t
        assert int(out[0]) == int(scratch[0])             # greedy: the megakernel's own token
        token = out.clone()
    assert sv.read_error()[0] == 0
    dec.close(), dec2.close(), sv.close()


def test_one_new_token_is_the_decoders_attention(etc):
    """The first layer's cache rows and the attention of a decode step, against the oracle's decode step on the same cache."""
    import oracle
    import synth
    from harness import GpuModel, fixed_step
    s = dataclasses.replace(synth.TINY_QK, n_layers=1)
    m = GpuModel(s, seed=5, n_pool_pages=32)
    step = fixed_step(s, 2, [130, 15], 32, seed=6)
    x = m.hidden(0, 2)
    w = m.weights[0]
    h = _norm(x.float(), w["g1"], s.eps)
    sv = etc.Serving(s, max_seqs=2, max_tokens=2, max_kv_len=256)
    table = np.zeros((2, 16), np.int32)
    for b in range(2):
        p = step.page_ids[step.page_indptr[b]:step.page_indptr[b + 1]]
        table[b, :len(p)] = p
    slots = [table[b, k // s.page] * s.page + k % s.page for b, k in enumerate(step.kv_len)]
    q_out, out = (torch.zeros(2, s.nq, s.d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.append(*(h @ w[n].float().t() for n in ("wq", "wk", "wv")), i32(step.kv_len), i32(slots), q_out, m.kpool[0], m.vpool[0], gq=w["gq"], gk=w["gk"])
    sv.attention(q_out, out, i32([0, 1, 2]), i32(step.kv_len), i32(table), m.kpool[0], m.vpool[0])
    y = x.float() + out.reshape(2, -1).float() @ w["wo"].float().t()
    g = _norm(y, w["g2"], s.eps)
    y = y + (torch.nn.functional.silu(g @ w["wg"].float().t()) * (g @ w["wu"].float().t())) @ w["wd"].float().t()
    res = oracle.decode_step(s, 1, synth.hidden_f32(s, 5, 0, 2), lambda l: synth.layer_weights_f32(s, 5, l),
                             lambda l: synth.kv_pool_f32(s, 5, l, 32), step)
    want = torch.as_tensor(res["final"])
    assert float((y.cpu() - want).abs().max() / want.pow(2).mean().sqrt()) < 2e-2      # the framework's bar
    sv.close()


def test_captured_step_follows_its_arrays(etc):
    """Tables, append, attention and sampling in one graph: replayed with other lengths, tables and inputs, with eager work of a
    second handle and synchronizations in between, every replay equal to the eager calls."""
    s = ref.shape(8, 2, 128, qk_norm=True, vocab=1500)
    n, rows, n_pages = 4, 600, 400
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *size, dtype=torch.bfloat16: torch.randn(*size, device="cuda", generator=g).to(dtype)        # noqa: E731
    svs = [etc.Serving(s, max_seqs=n, max_tokens=rows, max_kv_len=2000) for _ in range(2)]
    gq, gk = 1 + rnd(128), 1 + rnd(128)
    qkv, logits, u = rnd(rows, 12 * 128), rnd(n, 1500, dtype=torch.float32), torch.rand(n, device="cuda", generator=g)
    kv, new = i32([0, 0, 0, 0]), i32([1, 1, 1, 1])
    zero = lambda *size, dtype=torch.int32: torch.zeros(*size, dtype=dtype, device="cuda")        # noqa: E731

    def state():
        return {"table": zero(n, 125), "count": i32([n_pages]), "free": torch.arange(n_pages, dtype=torch.int32, device="cuda").flip(0).contiguous(),
                "q_indptr": zero(n + 1), "slots": zero(rows), "positions": zero(rows), "status": zero(1), "kv_after": zero(n), "count_after": zero(1),
                "q": zero(rows, 8, 128, dtype=torch.bfloat16), "out": zero(rows, 8, 128, dtype=torch.bfloat16), "token": zero(n),
                "lp": zero(n, dtype=torch.float32), "k": zero(n_pages, 16, 2, 128, dtype=torch.bfloat16), "v": zero(n_pages, 16, 2, 128, dtype=torch.bfloat16)}

    def step(sv, t):
        sv.tables(kv, new, t["table"], t["free"], t["count"], q_indptr=t["q_indptr"], slots=t["slots"], positions=t["positions"],
                  status=t["status"], free_count_out=t["count_after"], total_len=t["kv_after"])
        sv.append(qkv[:, :1024], qkv[:, 1024:1280], qkv[:, 1280:], t["positions"], t["slots"], t["q"], t["k"], t["v"], gq=gq, gk=gk)
        sv.attention(t["q"], t["out"], t["q_indptr"], kv, t["table"], t["k"], t["v"])
        sv.sample(logits, u, t["token"], top_p=zero(n, dtype=torch.float32) + 0.9, logprob_out=t["lp"])

    a, b = state(), state()
    step(svs[0], a)
    step(svs[1], b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(svs[0], a)
    for lens in ([3, 500, 0, 60], [1, 1, 1, 1], [0, 0, 0, 0], [256, 7, 30, 300], [2, 90, 100, 3]):
        new.copy_(i32(lens))
        qkv.copy_(rnd(rows, 12 * 128))
        logits.copy_(rnd(n, 1500, dtype=torch.float32))
        graph.replay()
        step(svs[1], b)
        torch.cuda.synchronize()
        for name in a:
            assert torch.equal(a[name], b[name]), (name, lens)
        assert int(a["status"]) == 0 and a["q_indptr"].tolist() == np.concatenate(([0], np.cumsum(lens))).tolist()
        kv.copy_(a["kv_after"])
        for t in (a, b):
            t["count"].copy_(t["count_after"])
        rnd(1 << 20).sum().item()
    assert kv.tolist() == [262, 598, 131, 364]
    for sv in svs:
        assert sv.read_error()[0] == 0
        sv.close()


def test_on_another_stream(etc):
    s = ref.shape(4, 2, 64)
    q, k, v = ref.randn(1, 40, 4, 64).cuda(), ref.randn(2, 9, 16, 2, 64).cuda(), ref.randn(3, 9, 16, 2, 64).cuda()
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    table = i32(np.arange(9)[None])
    sv = etc.Serving(s, max_seqs=1, max_tokens=40, max_kv_len=144)
    sv.attention(q, out, i32([0, 40]), i32([100]), table, k, v)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    qi, kv = i32([0, 40]), i32([100])
    torch.cuda.synchronize()
    sv.attention(q, again, qi, kv, table, k, v, stream=st)
    st.synchronize()
    assert torch.equal(out, again)
    sv.close()


def test_two_handles_at_once(etc):
    """Two handles on two streams, in turn and without waiting for each other: every call has its own workspace."""
    s = ref.shape(8, 2, 128, vocab=20000)
    q, k, v = ref.randn(1, 70, 8, 128).cuda(), ref.randn(2, 400, 16, 2, 128).cuda(), ref.randn(3, 400, 16, 2, 128).cuda()
    qi, kv, table = i32([0, 1, 70]), i32([3000, 3000]), i32(np.random.default_rng(1).permutation(400).reshape(2, 200))
    logits, u = ref.randn(4, 2, 20000, dtype=torch.float32).cuda(), torch.tensor([0.3, 0.9], device="cuda")
    svs = [etc.Serving(s, max_seqs=2, max_tokens=70, max_kv_len=3200) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    want, token = torch.zeros_like(q), i32([0, 0])
    svs[0].attention(q, want, qi, kv, table, k, v)
    svs[0].sample(logits, u, token)
    outs = [[torch.zeros_like(q) for _ in range(2)] for _ in range(8)]
    tokens = [[i32([-5, -5]) for _ in range(2)] for _ in range(8)]
    torch.cuda.synchronize()
    for i in range(8):
        for j in range(2):
            svs[j].attention(q, outs[i][j], qi, kv, table, k, v, stream=streams[j])
            svs[j].sample(logits, u, tokens[i][j], stream=streams[j])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for pair in outs for o in pair)
    assert all(torch.equal(t, token) for pair in tokens for t in pair)
    for sv in svs:
        assert sv.read_error()[0] == 0
        sv.close()


@pytest.mark.parametrize("vocab", [16383, 40001])
def test_captured_sampling_of_long_rows(etc, vocab):
    """One launch and three: replays with other logits and settings equal the eager calls of another handle."""
    s, n = ref.shape(vocab=vocab), 5
    g = torch.Generator(device="cuda").manual_seed(vocab)
    svs = [etc.Serving(s, max_seqs=n, max_tokens=1, max_kv_len=1) for _ in range(2)]
    x, u = torch.zeros(n, vocab, device="cuda"), torch.zeros(n, device="cuda")
    top_k, top_p = i32([0, 40, 1, 3000, 0]), torch.tensor([1.0, 0.9, 0.5, 0.99, 0.8], device="cuda")
    outs = [(i32([-5] * n), torch.zeros(n, device="cuda"), i32([-5] * n)) for _ in svs]

    def call(i):
        svs[i].sample(x, u, outs[i][0], top_k=top_k, top_p=top_p, logprob_out=outs[i][1], kept_out=outs[i][2])

    call(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0)
    for step in range(4):
        x.copy_(torch.randn(n, vocab, device="cuda", generator=g) * (0.5 + step))
        u.copy_(torch.rand(n, device="cuda", generator=g))
        top_k.copy_(top_k.roll(1))
        graph.replay()
        call(1)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs)), step
        assert int(outs[0][0].min()) >= 0
    for sv in svs:
        assert sv.read_error()[0] == 0
        sv.close()
