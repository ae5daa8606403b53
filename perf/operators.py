"""The operators around a decode step, as they are measured: page tables and slot maps made on the GPU, norms, rotation
and KV append of a chunk of new tokens, attention of a chunk over the paged cache, sampling of the next token.

A serving step is: `tables` once (requests' lengths in; pages, slots and positions out), per layer `append` (rows of the
QKV projection in; queries and cache rows out) and `attention`, and after the last layer `sample`.  A case is one call
of one of them.  `run` makes the framework's calls where `own` is true and computes the plain form otherwise.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

# (query heads, KV heads, head dim, per-head norms, rope theta, eps, vocabulary) of the framework's configurations
HEADS = {"tiny": (4, 2, 64, False, 1e4, 1e-5, 1024), "tiny-qk": (4, 2, 64, True, 1e4, 1e-5, 1024),
         "8b": (32, 8, 128, False, 1e4, 1e-5, 128256), "30b-a3b": (32, 4, 128, False, 1e4, 1e-5, 128256),
         "32b": (64, 8, 128, True, 1e6, 1e-6, 128256), "70b": (64, 8, 128, False, 1e4, 1e-5, 128256)}
PAGE = 16
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _tables(name, seqs, starting, chunk, longest, lens):
    return {"name": name, "op": "tables", "seqs": seqs, "starting": starting, "chunk": chunk, "longest": longest, "lens": lens}


def _append(name, shape, tokens, dtype, pad=0):
    return {"name": name, "op": "append", "shape": shape, "tokens": tokens, "pad": pad, "dtype": dtype}


def _attention(name, shape, seqs, starting, chunk, few, longest, lens):
    return {"name": name, "op": "attention", "shape": shape, "seqs": seqs, "starting": starting, "chunk": chunk, "few": few,
            "longest": longest, "lens": lens}


def _sample(name, rows, vocab, dtype, mode):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "mode": mode}


def listed():
    return [
        # three requests that decode, one token each: a launch is all there is
        _tables("tables_3", 3, 0, 1, 300, 1),
        # a loaded server: 200 requests, 20 of them with a chunk of their prompt, long contexts
        _tables("tables_200", 200, 20, 2000, 16000, 2),
        # a few decoding requests of the smallest model
        _append("append_3", "tiny-qk", 3, "bf16"),
        # an ordinary chunk of a prompt without norms, fp32 projections, in a buffer padded to a fixed size
        _append("append_1000", "8b", 1000, "fp32", 24),
        # the largest chunk, per-head norms
        _append("append_8192", "32b", 8192, "bf16"),
        # three short sequences of the smallest model, one token each
        _attention("attn_few", "tiny", 3, 0, 1, 1, 300, 3),
        # 16 requests whose last few tokens are checked together, odd context lengths
        _attention("attn_verify_16", "8b", 16, 0, 1, 5, 4100, 4),
        # a mixed step: two prompts under way among 30 decoding requests
        _attention("attn_mixed_32", "30b-a3b", 32, 2, 1500, 1, 4096, 5),
        # a long prompt: its last chunk over all the chunks before it
        _attention("attn_long", "70b", 1, 1, 4001, 1, 30000, 6),
        # one user, usual settings, a small vocabulary
        _sample("sample_1_small", 1, 1024, "fp32", "both"),
        # a step of 16 requests without filters: the draw goes over the whole vocabulary
        _sample("sample_16_open", 16, 128256, "fp32", "open"),
        # a full batch, every request with its own settings, 16-bit logits with ties, banned tokens
        _sample("sample_64_mixed", 64, 128256, "bf16", "mixed"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "append", "attention", "attention", "sample"])
    if op == "tables":
        seqs = _spread(rng, 1, 256)
        c = _tables("", seqs, rng.randint(0, min(seqs, 20)), _spread(rng, 1, 2000), _spread(rng, 16, 16000), rng.randrange(1 << 20))
    elif op == "append":
        c = _append("", rng.choice(sorted(HEADS)), _spread(rng, 1, 8192), rng.choice(["bf16", "fp32"]), rng.choice([0, 0, 7, 100]))
    elif op == "sample":
        c = _sample("", _spread(rng, 1, 64), rng.choice([1024, 128256, _spread(rng, 100, 128256)]), rng.choice(["bf16", "fp32"]),
                    rng.choice(["open", "top_k", "top_p", "both", "mixed"]))
    else:
        while True:
            seqs = _spread(rng, 1, 128)
            c = _attention("", rng.choice(["tiny", "8b", "30b-a3b", "32b", "70b"]), seqs, rng.randint(0, min(seqs, 4)),
                           _spread(rng, 1, 8192), _spread(rng, 1, 8), _spread(rng, 16, 32768), rng.randrange(1 << 20))
            w = work(c)
            if w["flops"] <= 4.5e12 and w["bytes"] <= 4e9:
                break
    del c["name"]
    return c


# ---- lengths: plain values of the case --------------------------------------------------------------------------------
def _lengths(case):
    """(cached tokens, new tokens) of every sequence.  The sequences that process their prompt come at odd places among
    the others; one alone has the lengths of the case, several are ragged."""
    rng = random.Random(case["lens"])
    n, few = case["seqs"], case.get("few", 1)
    at = set(rng.sample(range(n), case["starting"]))
    kv, new = [], []
    for i in range(n):
        kv.append(case["longest"] if n == 1 else rng.randint(case["longest"] // 2, case["longest"]))
        if i in at:
            new.append(case["chunk"] if n == 1 else rng.randint((case["chunk"] + 1) // 2, case["chunk"]))
            if rng.random() < 0.5 and n > 1:
                kv[-1] = 0                                     # its first chunk
        else:
            new.append(few if case["op"] == "attention" else rng.choice([1, 1, 1, 0]) if n > 4 else 1)
    return kv, new


def _pages(tokens):
    return -(-tokens // PAGE)


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype=torch.bfloat16, sigma=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _block_table(g, owned):
    """Random pages: [sequence][page] and the ids nobody owns."""
    total = sum(owned) + sum(owned) // 8 + 8
    perm = torch.randperm(total, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros(len(owned), max(owned) + 1, dtype=torch.int32, device="cuda")
    rows = torch.repeat_interleave(torch.arange(len(owned)), torch.tensor(owned))
    cols = torch.cat([torch.arange(n) for n in owned])
    table[rows.cuda(), cols.cuda()] = perm[:sum(owned)]
    return table, perm[sum(owned):].contiguous(), total


def _inputs(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "tables":
        kv, new = _lengths(case)
        has, need = [_pages(k) for k in kv], [_pages(k + n) for k, n in zip(kv, new)]
        table, rest, total = _block_table(g, has)
        wide = torch.zeros(len(kv), max(max(need), 1) + 3, dtype=torch.int32, device="cuda")
        w = min(wide.shape[1], table.shape[1])
        wide[:, :w] = table[:, :w]
        missing = sum(need) - sum(has)
        fresh = torch.arange(total, total + missing + 5, dtype=torch.int32, device="cuda")
        free = torch.cat((rest, fresh))
        free = free[torch.randperm(free.numel(), device="cuda", generator=g)].contiguous()
        return SimpleNamespace(case=case, kv=kv, new=new, kv_len=_ints(kv), new_len=_ints(new), table=wide, free=free,
                               free_count=_ints([free.numel()]), tokens=sum(new), ids=sum(need))
    if op == "append":
        nq, nkv, d, norm, theta, eps, _ = HEADS[case["shape"]]
        rows, pages = case["tokens"] + case["pad"], _pages(case["tokens"]) + 4
        qkv = _normal(g, (rows, (nq + 2 * nkv) * d), DTYPE[case["dtype"]])
        slots = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        page = torch.randperm(pages, device="cuda", generator=g)
        t = torch.arange(case["tokens"], device="cuda")
        slots[:case["tokens"]] = (page[t // PAGE] * PAGE + t % PAGE).to(torch.int32)
        positions = torch.zeros(rows, dtype=torch.int32, device="cuda")
        positions[:case["tokens"]] = (t + int(torch.randint(0, 30000, (1,), device="cuda", generator=g))).to(torch.int32)
        i = SimpleNamespace(case=case, qkv=qkv, slots=slots, positions=positions, gq=None, gk=None,
                            k=_normal(g, (pages, PAGE, nkv, d)), v=_normal(g, (pages, PAGE, nkv, d)),
                            q_out=torch.zeros(rows, nq, d, dtype=torch.bfloat16, device="cuda"))
        if norm:
            i.gq, i.gk = (1.0 + 0.25 * _normal(g, (d,), torch.float32)).bfloat16(), (1.0 + 0.25 * _normal(g, (d,), torch.float32)).bfloat16()
        return i
    if op == "attention":
        nq, nkv, d = HEADS[case["shape"]][:3]
        kv, new = _lengths(case)
        table, _, total = _block_table(g, [_pages(k + n) for k, n in zip(kv, new)])
        indptr = [0]
        for n in new:
            indptr.append(indptr[-1] + n)
        return SimpleNamespace(case=case, kv=kv, new=new, indptr=indptr, q=_normal(g, (indptr[-1], nq, d)), table=table,
                               kv_len=_ints(kv), q_indptr=_ints(indptr), k=_normal(g, (total, PAGE, nkv, d)),
                               v=_normal(g, (total, PAGE, nkv, d)), out=torch.zeros(indptr[-1], nq, d, dtype=torch.bfloat16, device="cuda"))
    rows, vocab, mode = case["rows"], case["vocab"], case["mode"]
    x = _normal(g, (rows, vocab), torch.float32, 2.5)
    best = torch.randint(0, vocab, (rows, 24), device="cuda", generator=g)           # a few likely tokens stand out
    x.scatter_add_(1, best, 6.0 + _normal(g, (rows, 24), torch.float32, 2.0))
    if mode == "mixed":
        x.masked_fill_(torch.rand(rows, vocab, device="cuda", generator=g) < 0.05, -math.inf)
    pick = lambda values: torch.tensor(values, device="cuda")[torch.randint(0, len(values), (rows,), device="cuda", generator=g)]  # noqa: E731
    i = SimpleNamespace(case=case, logits=x.to(DTYPE[case["dtype"]]), u=torch.rand(rows, device="cuda", generator=g),
                        temperature=None, top_k=None, top_p=None, min_p=None,
                        token=torch.zeros(rows, dtype=torch.int32, device="cuda"), logprob=torch.zeros(rows, device="cuda"),
                        kept=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    i.temperature = pick([0.0, 0.6, 0.8, 1.0, 1.3] if mode == "mixed" else [0.7, 1.0])
    if mode in ("top_k", "both", "mixed"):
        i.top_k = pick([0, 1, 20, 50, 1000] if mode == "mixed" else [20, 50]).to(torch.int32)
    if mode in ("top_p", "both", "mixed"):
        i.top_p = pick([1.0, 0.95, 0.9, 0.5] if mode == "mixed" else [0.95, 0.9])
    if mode == "mixed":
        i.min_p = pick([0.0, 0.0, 0.05, 0.2])
    return i


def prepare(case, seed):
    i = _inputs(case, seed)
    if own:
        import paper_2604_13327_amd as etc
        nq, nkv, d, norm, theta, eps, vocab = HEADS[case.get("shape", "tiny")]
        shape = SimpleNamespace(n_layers=1, H=nq * d, nq=nq, nkv=nkv, d=d, F=0, n_experts=0, top_k=0, moe_F=0, page=PAGE, eps=eps,
                                theta=theta, qk_norm=norm, vocab=case.get("vocab", vocab))
        if case["op"] in ("tables", "attention"):
            seqs, tokens, longest = len(i.kv), sum(i.new) + 3, max(k + n for k, n in zip(i.kv, i.new))
        elif case["op"] == "append":
            seqs, tokens, longest = 1, case["tokens"] + case["pad"], 65536
        else:
            seqs, tokens, longest = case["rows"], case["rows"], 1
        i.serving = etc.Serving(shape, max_seqs=seqs, max_tokens=tokens, max_kv_len=longest)
    if case["op"] == "tables":
        n, e = case["seqs"], lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")      # noqa: E731
        i.out = {"block_table": i.table, "free_count": e(1), "q_indptr": e(n + 1), "slots": e(i.tokens + 3),
                 "positions": e(i.tokens + 3), "total_len": e(n), "page_indptr": e(n + 1), "page_ids": e(i.ids), "status": e(1)}
    return i


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(i):
    return {"tables": _run_tables, "append": _run_append, "attention": _run_attention, "sample": _run_sample}[i.case["op"]](i)


def _run_tables(i):
    o = i.out
    if own:
        i.serving.tables(i.kv_len, i.new_len, o["block_table"], i.free, i.free_count, q_indptr=o["q_indptr"], slots=o["slots"],
                         positions=o["positions"], status=o["status"], free_count_out=o["free_count"], total_len=o["total_len"],
                         page_indptr=o["page_indptr"], page_ids=o["page_ids"])
        return o
    kv, new, dev = i.kv_len.long(), i.new_len.long(), i.kv_len.device
    total = kv + new
    has, need = (kv + PAGE - 1) // PAGE, (total + PAGE - 1) // PAGE
    first_new = torch.cumsum(need - has, 0) - (need - has)                       # taken by the sequences before
    o["total_len"].copy_(total)
    o["q_indptr"][1:] = torch.cumsum(new, 0)
    o["page_indptr"][1:] = torch.cumsum(need, 0)
    o["free_count"].copy_(i.free_count - (need - has).sum())
    o["status"].zero_()
    page = torch.arange(o["block_table"].shape[1], device=dev)[None, :]
    taken = (page >= has[:, None]) & (page < need[:, None])
    rank = (i.free_count.long() - 1 - first_new[:, None] - (page - has[:, None])).clamp(0, i.free.numel() - 1)
    o["block_table"].copy_(torch.where(taken, i.free[rank], o["block_table"]))
    o["page_ids"].copy_(o["block_table"][page.expand_as(taken) < need[:, None]])
    row = torch.arange(o["slots"].numel(), device=dev)
    seq = (torch.searchsorted(o["q_indptr"].long(), row, right=True) - 1).clamp(max=kv.numel() - 1)
    pos = kv[seq] + row - o["q_indptr"].long()[seq]
    live = row < o["q_indptr"][-1]
    at = o["block_table"][seq, (pos // PAGE).clamp(0, o["block_table"].shape[1] - 1)].long() * PAGE + pos % PAGE
    o["slots"].copy_(torch.where(live, at, -1))
    o["positions"].copy_(torch.where(live, pos, 0))
    return o


def _rotate(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)


def _heads(i):
    nq, nkv, d, norm, theta, eps, _ = HEADS[i.case["shape"]]
    return nq, nkv, d, norm, theta, eps


def _run_append(i):
    nq, nkv, d, norm, theta, eps = _heads(i)
    q, k, v = i.qkv[:, :nq * d], i.qkv[:, nq * d:(nq + nkv) * d], i.qkv[:, (nq + nkv) * d:]
    if own:
        i.serving.append(q, k, v, i.positions, i.slots, i.q_out, i.k, i.v, gq=i.gq, gk=i.gk)
        return {"q": i.q_out, "k": i.k, "v": i.v}
    rows = i.slots.shape[0]
    q, k, v = (t.float().reshape(rows, -1, d) for t in (q, k, v))
    if norm:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + eps) * i.gq.float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + eps) * i.gk.float()
    ang = i.positions.double()[:, None] * theta ** (-2.0 * torch.arange(d // 2, device=q.device).double() / d)
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    live = i.slots >= 0
    at = i.slots[live].long()
    i.q_out.copy_(torch.where(live[:, None, None], _rotate(q, cos, sin).bfloat16(), i.q_out))
    i.k.view(-1, nkv, d)[at] = _rotate(k, cos, sin)[live].bfloat16()
    i.v.view(-1, nkv, d)[at] = v[live].bfloat16()
    return {"q": i.q_out, "k": i.k, "v": i.v}


def _run_attention(i):
    if own:
        i.serving.attention(i.q, i.out, i.q_indptr, i.kv_len, i.table, i.k, i.v)
        return i.out
    nq, nkv, d = HEADS[i.case["shape"]][:3]
    for b, (kv, new) in enumerate(zip(i.kv, i.new)):
        if new == 0:
            continue
        total = kv + new
        pages = i.table[b, :_pages(total)].long()
        k, v = (p[pages].reshape(-1, nkv, d)[:total].float().transpose(0, 1).contiguous() for p in (i.k, i.v))
        kt = k.transpose(1, 2).contiguous()
        step = max(1, (1 << 28) // (nq * total))
        for r in range(0, new, step):
            n = min(step, new - r)
            q = i.q[i.indptr[b] + r:i.indptr[b] + r + n].float().view(n, nkv, nq // nkv, d).permute(1, 2, 0, 3).reshape(nkv, -1, d)
            score = (torch.bmm(q.contiguous(), kt) / math.sqrt(d)).view(nkv, nq // nkv, n, total)
            late = torch.arange(total, device=q.device)[None, :] > kv + r + torch.arange(n, device=q.device)[:, None]
            score.masked_fill_(late, -math.inf)
            score -= score.amax(-1, keepdim=True)
            score.exp_()
            norm = score.sum(-1, keepdim=True)
            o = torch.bmm(score.view(nkv, -1, total), v).view(nkv, nq // nkv, n, d) / norm
            i.out[i.indptr[b] + r:i.indptr[b] + r + n] = o.permute(2, 0, 1, 3).reshape(n, nq, d).bfloat16()
    return i.out


def _run_sample(i):
    if own:
        i.serving.sample(i.logits, i.u, i.token, temperature=i.temperature, top_k=i.top_k, top_p=i.top_p, min_p=i.min_p,
                         logprob_out=i.logprob, kept_out=i.kept)
        return {"token": i.token, "logprob": i.logprob, "kept": i.kept}
    x = i.logits.double()
    rows, vocab = x.shape
    first = x.max(-1, keepdim=True)
    x, order = x.sort(dim=-1, descending=True, stable=True)
    temperature = i.temperature.double()[:, None]
    w = torch.exp((x - first.values) / torch.where(temperature > 0, temperature, 1.0))
    rank = torch.arange(vocab, device=x.device)[None, :]
    if i.top_k is not None:
        k = i.top_k.long()[:, None]
        w = torch.where((rank < k) | (k <= 0), w, 0.0)
    keep = x > -math.inf
    if i.top_k is not None:
        keep &= (rank < k) | (k <= 0)
    if i.top_p is not None:
        p = i.top_p.double()[:, None]
        before = torch.cumsum(w, -1) - w
        keep &= (before < p * w.sum(-1, keepdim=True)) | (p >= 1) | (rank == 0)
    if i.min_p is not None:
        keep &= (w >= i.min_p.double()[:, None]) | (rank == 0)
    w = torch.where(keep, w, 0.0)
    up_to = torch.cumsum(w, -1)
    drawn = (up_to <= i.u.double()[:, None] * up_to[:, -1:]).sum(-1).clamp(max=vocab - 1)
    drawn = torch.minimum(drawn, keep.sum(-1) - 1)
    greedy = ~(temperature[:, 0] > 0)
    drawn = torch.where(greedy, 0, drawn)[:, None]
    i.token.copy_(order.gather(1, drawn)[:, 0])
    i.logprob.copy_(torch.where(greedy, 0.0, torch.log(w.gather(1, drawn) / up_to[:, -1:])[:, 0]))
    i.kept.copy_(torch.where(greedy, 1, keep.sum(-1)))
    return {"token": i.token, "logprob": i.logprob, "kept": i.kept}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "tables":
        kv, new = _lengths(case)
        need, tokens = sum(_pages(k + n) for k, n in zip(kv, new)), sum(new)
        fresh = need - sum(_pages(k) for k in kv)
        # lengths in, three index arrays and the totals out; slots and positions out; pages read and written, fresh ones into the table
        return {"bytes": 4 * (2 * len(kv) + 3 * len(kv) + 2 + 2 * (tokens + 3) + 2 * need + fresh), "flops": 2 * tokens + need}
    if case["op"] == "append":
        nq, nkv, d, norm = HEADS[case["shape"]][:4]
        size = 4 if case["dtype"] == "fp32" else 2
        n = case["tokens"] * (nq + 2 * nkv) * d
        return {"bytes": n * (size + 2) + 8 * (case["tokens"] + case["pad"]), "flops": case["tokens"] * (nq + nkv) * d * (7 if norm else 3)}
    if case["op"] == "attention":
        nq, nkv, d = HEADS[case["shape"]][:3]
        kv, new = _lengths(case)
        pairs = sum(n * k + n * (n + 1) // 2 for k, n in zip(kv, new))
        keys = sum(k + n for k, n in zip(kv, new) if n)
        return {"bytes": 4 * sum(new) * nq * d + 4 * keys * nkv * d, "flops": 4 * pairs * nq * d}
    size = 4 if case["dtype"] == "fp32" else 2
    return {"bytes": case["rows"] * (case["vocab"] * size + 32), "flops": 4 * case["rows"] * case["vocab"]}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    i = _inputs(case, seed)
    return {"tables": _exact_tables, "append": _exact_append, "attention": _exact_attention, "sample": _exact_sample}[case["op"]](i)


def _exact_tables(i):
    table, free = i.table.cpu().tolist(), i.free.cpu().tolist()
    q_indptr, page_indptr, slots, positions, ids = [0], [0], [], [], []
    for b, (kv, new) in enumerate(zip(i.kv, i.new)):
        for p in range(_pages(kv), _pages(kv + new)):
            table[b][p] = free.pop()
        for pos in range(kv, kv + new):
            slots.append(table[b][pos // PAGE] * PAGE + pos % PAGE)
            positions.append(pos)
        ids += table[b][:_pages(kv + new)]
        q_indptr.append(len(slots))
        page_indptr.append(len(ids))
    return {"block_table": _ints(table), "free_count": _ints([len(free)]), "q_indptr": _ints(q_indptr), "slots": _ints(slots + [-1] * 3),
            "positions": _ints(positions + [0] * 3), "total_len": _ints([k + n for k, n in zip(i.kv, i.new)]),
            "page_indptr": _ints(page_indptr), "page_ids": _ints(ids), "status": _ints([0])}


def _exact_append(i):
    nq, nkv, d, norm, theta, eps = _heads(i)
    live = (i.slots >= 0).nonzero()[:, 0]
    x = i.qkv[live].double().view(live.numel(), nq + 2 * nkv, d)
    heads, v = x[:, :nq + nkv].clone(), x[:, nq + nkv:]
    if norm:
        gain = torch.cat((i.gq.double().expand(nq, d), i.gk.double().expand(nkv, d)))
        heads = heads / torch.sqrt(heads.pow(2).sum(-1, keepdim=True) / d + eps) * gain
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device=x.device),
                       i.positions[live].double()[:, None] * torch.exp(torch.arange(d // 2, device=x.device).double() * (-2.0 * math.log(theta) / d)))
    pair = torch.complex(heads[..., :d // 2].contiguous(), heads[..., d // 2:].contiguous()) * turn[:, None]
    heads = torch.cat((pair.real, pair.imag), -1)
    q, k, vv = i.q_out.double(), i.k.double(), i.v.double()
    q[live] = heads[:, :nq]
    page, off = i.slots[live].long() // PAGE, i.slots[live].long() % PAGE
    k[page, off] = heads[:, nq:]
    vv[page, off] = v
    return {"q": q, "k": k, "v": vv}


def _exact_attention(i):
    nq, nkv, d = HEADS[i.case["shape"]][:3]
    out = torch.zeros(i.indptr[-1], nq, d, dtype=torch.float64, device="cuda")
    for b, (kv, new) in enumerate(zip(i.kv, i.new)):
        slot = torch.arange(kv + new, device="cuda")
        page = i.table[b].long()[slot // PAGE]
        for h in range(nkv):
            k, v = i.k[page, slot % PAGE, h].double(), i.v[page, slot % PAGE, h].double()
            for g in range(h * (nq // nkv), (h + 1) * (nq // nkv)):
                for r in range(0, new, 2048):
                    q = i.q[i.indptr[b] + r:min(i.indptr[b] + r + 2048, i.indptr[b + 1]), g].double()
                    seen = slot[None, :] <= kv + r + torch.arange(q.shape[0], device="cuda")[:, None]
                    p = torch.where(seen, (q @ k.t()) * d ** -0.5, -math.inf).softmax(-1)
                    out[i.indptr[b] + r:i.indptr[b] + r + q.shape[0], g] = p @ v
    return out


def _exact_sample(i):
    tokens, logprobs, kept = [], [], []
    settings = [None if t is None else t.tolist() for t in (i.temperature, i.top_k, i.top_p, i.min_p)]
    for row, u in enumerate(i.u.tolist()):
        temperature, top_k, top_p, min_p = (default if s is None else s[row] for s, default in zip(settings, (1.0, 0, 1.0, 0.0)))
        x = i.logits[row].double()
        ids = torch.argsort(x, descending=True, stable=True)
        if not temperature > 0:
            tokens.append(int(ids[0]))
            logprobs.append(0.0)
            kept.append(1)
            continue
        ids = ids[:int((x > -math.inf).sum())]
        if top_k > 0:
            ids = ids[:top_k]
        z = x[ids] / temperature
        mass = torch.cumsum(torch.softmax(z, 0), 0)
        n = ids.numel()
        if top_p < 1:
            n = min(n, int((mass < top_p * mass[-1]).sum()) + 1)
        if min_p > 0:
            n = min(n, max(1, int((torch.exp(z - z[0]) >= min_p).sum())))
        p = torch.softmax(z[:n], 0)
        at = min(int((torch.cumsum(p, 0) <= u).sum()), n - 1)
        tokens.append(int(ids[at]))
        logprobs.append(float(torch.log_softmax(z[:n], 0)[at]))
        kept.append(n)
    return {"token": _ints(tokens), "logprob": torch.tensor(logprobs, dtype=torch.float64, device="cuda"), "kept": _ints(kept)}
