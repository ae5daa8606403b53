"""The operators of a cache held in 8 bits, and of scores, as they are measured: norms, rotation and append of a chunk of new
tokens to a paged cache of e4m3 codes with a power of two for each page and KV head, attention of a chunk over that cache, and log
probabilities of given tokens with entropy and the likeliest alternatives.

A step of a server that keeps its cache in 8 bits calls, per layer, `append_codes` (rows of the QKV projection in; queries, codes and
scales out) and `attention_codes`; a request that asks for log probabilities has `score` over its rows of logits.  A case is one call
of one of them.  `run` makes the framework's calls where `own` is true and computes the plain form otherwise.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

# (query heads, KV heads, head dim, per-head norms, rope theta, eps) of the framework's configurations
HEADS = {"tiny": (4, 2, 64, False, 1e4, 1e-5), "tiny-qk": (4, 2, 64, True, 1e4, 1e-5), "8b": (32, 8, 128, False, 1e4, 1e-5),
         "30b-a3b": (32, 4, 128, False, 1e4, 1e-5), "32b": (64, 8, 128, True, 1e6, 1e-6), "70b": (64, 8, 128, False, 1e4, 1e-5)}
PAGE = 16
LOWEST = -40                # exponent of a scale
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _append(name, shape, seqs, starting, chunk, dtype, pad, longest, lens):
    return {"name": name, "op": "append", "shape": shape, "seqs": seqs, "starting": starting, "chunk": chunk, "few": 1, "dtype": dtype,
            "pad": pad, "longest": longest, "lens": lens}


def _attention(name, shape, seqs, starting, chunk, few, longest, lens):
    return {"name": name, "op": "attention", "shape": shape, "seqs": seqs, "starting": starting, "chunk": chunk, "few": few,
            "longest": longest, "lens": lens}


def _score(name, rows, vocab, dtype, top, banned):
    return {"name": name, "op": "score", "rows": rows, "vocab": vocab, "dtype": dtype, "top": top, "banned": banned}


def listed():
    return [
        # three decoding requests of the smallest model, in pages begun: a launch is all there is
        _append("append_3", "tiny-qk", 3, 0, 1, "bf16", 0, 300, 1),
        # a loaded server's decode step, every request in another page, fp32 projections in a padded buffer
        _append("append_200", "8b", 200, 0, 1, "fp32", 56, 8000, 2),
        # an ordinary chunk of one prompt behind an odd number of cached tokens
        _append("append_1000", "8b", 1, 1, 1000, "bf16", 24, 333, 3),
        # the largest step: prompts of several requests, per-head norms
        _append("append_7328", "32b", 12, 4, 2600, "bf16", 0, 4000, 5),
        # three short sequences of the smallest model, one token each
        _attention("attn_few", "tiny", 3, 0, 1, 1, 300, 3),
        # a decode step of 64 requests over long contexts: the cache's bytes
        _attention("attn_decode_64", "8b", 64, 0, 1, 1, 8000, 4),
        # a mixed step: two prompts under way among 30 decoding requests
        _attention("attn_mixed_32", "30b-a3b", 32, 2, 1500, 1, 4096, 5),
        # a long prompt: its last chunk over all the chunks before it
        _attention("attn_long", "70b", 1, 1, 4001, 1, 30000, 6),
        # one user, a small vocabulary
        _score("score_1_small", 1, 1024, "fp32", 5, False),
        # a decode step of 16 requests that ask for the 20 likeliest tokens
        _score("score_16", 16, 128256, "fp32", 20, False),
        # a batch whose sampler has banned tokens, 16-bit logits with ties
        _score("score_301_banned", 301, 128256, "bf16", 10, True),
        # a prompt's log probabilities
        _score("score_4096", 4096, 128256, "bf16", 5, False),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "score"])
    while True:
        if op == "append":
            seqs = _spread(rng, 1, 256)
            c = _append("", rng.choice(sorted(HEADS)), seqs, rng.randint(0, min(seqs, 6)), _spread(rng, 1, 8192), rng.choice(["bf16", "fp32"]),
                        rng.choice([0, 0, 7, 100]), _spread(rng, 1, 30000), rng.randrange(1 << 20))
            if sum(_lengths(c)[1]) <= (8192 if c["dtype"] == "bf16" else 4096):
                break
        elif op == "attention":
            seqs = _spread(rng, 1, 128)
            c = _attention("", rng.choice(sorted(HEADS)), seqs, rng.randint(0, min(seqs, 4)), _spread(rng, 1, 8192), _spread(rng, 1, 8),
                           _spread(rng, 16, 32768), rng.randrange(1 << 20))
            w = work(c)
            if w["flops"] <= 4.2e12 and w["bytes"] <= 2.2e9:
                break
        else:
            c = _score("", _spread(rng, 1, 4096), rng.choice([1024, 128256, _spread(rng, 100, 128256)]), rng.choice(["bf16", "fp32"]),
                       rng.choice([1, 5, 20, rng.randint(1, 64)]), rng.random() < 0.3)
            if work(c)["bytes"] <= 1.05e9:
                break
    del c["name"]
    return c


# ---- lengths: plain values of the case --------------------------------------------------------------------------------
def _lengths(case):
    """(cached tokens, new tokens) of every sequence.  The sequences that process their prompt come at odd places among
    the others; one alone has the lengths of the case, several are ragged."""
    rng = random.Random(case["lens"])
    n = case["seqs"]
    at = set(rng.sample(range(n), case["starting"]))
    kv, new = [], []
    for i in range(n):
        kv.append(case["longest"] if n == 1 else rng.randint(case["longest"] // 2, case["longest"]))
        if i in at:
            new.append(case["chunk"] if n == 1 else rng.randint((case["chunk"] + 1) // 2, case["chunk"]))
            if rng.random() < 0.5 and n > 1:
                kv[-1] = 0                                     # its first chunk
        else:
            new.append(case["few"])
    return kv, new


def _pages(tokens):
    return -(-tokens // PAGE)


def _touched(kv, new):
    """Pages that the new tokens of a sequence lie in."""
    return _pages(kv + new) - kv // PAGE


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype=torch.bfloat16, sigma=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache(g, pages, nkv, d):
    """Pages in use: codes and scales as values of about 1, a quarter or a sixteenth by page and head leave them."""
    shift = torch.randint(0, 3, (pages, nkv), device="cuda", generator=g) * 2
    codes = _normal(g, (pages, PAGE, nkv, d), torch.float32, 80.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
    return codes, (127 - 6 - shift).to(torch.uint8).view(torch.float8_e8m0fnu)


def _inputs(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "append":
        nq, nkv, d, norm = HEADS[case["shape"]][:4]
        kv, new = _lengths(case)
        tokens, each = sum(new), [_touched(k, n) for k, n in zip(kv, new)]
        rows, pages = tokens + case["pad"], sum(each) + 5
        perm, slots, positions, at = torch.randperm(pages, device="cuda", generator=g), [], [], 0
        for k, n, m in zip(kv, new, each):
            t = torch.arange(k, k + n, device="cuda")
            slots.append(perm[at + t // PAGE - k // PAGE] * PAGE + t % PAGE)
            positions.append(t)
            at += m
        pad = torch.full((case["pad"],), -1, device="cuda")
        i = SimpleNamespace(case=case, qkv=_normal(g, (rows, (nq + 2 * nkv) * d), DTYPE[case["dtype"]]), gq=None, gk=None,
                            slots=torch.cat(slots + [pad]).to(torch.int32), positions=torch.cat(positions + [pad * 0]).to(torch.int32),
                            q_out=torch.zeros(rows, nq, d, dtype=torch.bfloat16, device="cuda"))
        i.k, i.ks = _cache(g, pages, nkv, d)
        i.v, i.vs = _cache(g, pages, nkv, d)
        if norm:
            i.gq, i.gk = (1.0 + 0.25 * _normal(g, (d,), torch.float32)).bfloat16(), (1.0 + 0.25 * _normal(g, (d,), torch.float32)).bfloat16()
        return i
    if op == "attention":
        nq, nkv, d = HEADS[case["shape"]][:3]
        kv, new = _lengths(case)
        owned = [_pages(k + n) for k, n in zip(kv, new)]
        total = sum(owned) + sum(owned) // 8 + 8
        table = torch.zeros(len(owned), max(owned) + 1, dtype=torch.int32, device="cuda")
        rows = torch.repeat_interleave(torch.arange(len(owned)), torch.tensor(owned))
        table[rows.cuda(), torch.cat([torch.arange(n) for n in owned]).cuda()] = torch.randperm(total, device="cuda", generator=g)[:sum(owned)].to(torch.int32)
        indptr = [0]
        for n in new:
            indptr.append(indptr[-1] + n)
        i = SimpleNamespace(case=case, kv=kv, new=new, indptr=indptr, q=_normal(g, (indptr[-1], nq, d)), table=table, kv_len=_ints(kv),
                            q_indptr=_ints(indptr), out=torch.zeros(indptr[-1], nq, d, dtype=torch.bfloat16, device="cuda"))
        i.k, i.ks = _cache(g, total, nkv, d)
        i.v, i.vs = _cache(g, total, nkv, d)
        return i
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    x = _normal(g, (rows, vocab), torch.float32, 2.5)
    best = torch.randint(0, vocab, (rows, 24), device="cuda", generator=g)           # a few likely tokens stand out
    x.scatter_add_(1, best, 6.0 + _normal(g, (rows, 24), torch.float32, 2.0))
    if case["banned"]:
        x.masked_fill_(torch.rand(rows, vocab, device="cuda", generator=g) < 0.05, -math.inf)
    tokens = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.7, best[:, 0], torch.randint(0, vocab, (rows,), device="cuda", generator=g))
    return SimpleNamespace(case=case, logits=x.to(DTYPE[case["dtype"]]), tokens=tokens.to(torch.int32), logprob=torch.zeros(rows, device="cuda"),
                           entropy=torch.zeros(rows, device="cuda"), top_ids=torch.zeros(rows, top, dtype=torch.int32, device="cuda"),
                           top_logprobs=torch.zeros(rows, top, device="cuda"))


def prepare(case, seed):
    i = _inputs(case, seed)
    if own:
        import paper_2604_13327_amd as etc
        nq, nkv, d, norm, theta, eps = HEADS[case.get("shape", "tiny")]
        shape = SimpleNamespace(n_layers=1, H=nq * d, nq=nq, nkv=nkv, d=d, F=0, n_experts=0, top_k=0, moe_F=0, page=PAGE, eps=eps,
                                theta=theta, qk_norm=norm, vocab=case.get("vocab", 0))
        if case["op"] == "append":
            seqs, tokens, longest = case["seqs"], i.slots.numel(), 65536
        elif case["op"] == "attention":
            seqs, tokens, longest = case["seqs"], i.indptr[-1], max(k + n for k, n in zip(i.kv, i.new))
        else:
            seqs, tokens, longest = min(case["rows"], 256), case["rows"], 1
        i.serving = etc.Serving(shape, max_seqs=seqs, max_tokens=tokens, max_kv_len=longest)
    return i


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(i):
    return {"append": _run_append, "attention": _run_attention, "score": _run_score}[i.case["op"]](i)


def _rotate(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)


def _store(x, slots, codes, scale):
    """Values x [rows, heads, d] to the slots of a pool: new scales of the pages, codes of all of a page's tokens up to the last new one."""
    pages, _, nkv, d = codes.shape
    page, off = slots // PAGE, slots % PAGE
    first = torch.full((pages,), PAGE, device=x.device).scatter_reduce(0, page, off, "amin")
    last = torch.full((pages,), -1, device=x.device).scatter_reduce(0, page, off, "amax")
    size = torch.zeros(pages, nkv, device=x.device).scatter_reduce(0, page[:, None].expand(-1, nkv), x.abs().amax(-1), "amax")
    # the smallest power of two whose 448 times reach it
    part, power = torch.frexp(size)
    need = torch.where(size > 0, (power - 9 + (part > 0.875)).clamp(min=LOWEST), LOWEST)
    before = scale.view(torch.uint8).int() - 127
    after = torch.where(first[:, None] > 0, torch.maximum(before, need), need)
    after = torch.where(last[:, None] >= 0, after, before)
    index = torch.arange(PAGE, device=x.device)
    kept = (index[None, :] < first[:, None]) & (last[:, None] >= 0)
    old = codes.float() * torch.exp2((before - after).float())[:, None, :, None]
    codes.copy_(torch.where(kept[:, :, None, None], old.to(codes.dtype).float(), codes.float()).to(codes.dtype))
    codes.view(-1, nkv, d)[slots] = (x * torch.exp2(-after[page].float())[:, :, None]).to(codes.dtype)
    scale.view(torch.uint8).copy_((after + 127).to(torch.uint8))


def _run_append(i):
    nq, nkv, d, norm, theta, eps = HEADS[i.case["shape"]]
    q, k, v = i.qkv[:, :nq * d], i.qkv[:, nq * d:(nq + nkv) * d], i.qkv[:, (nq + nkv) * d:]
    if own:
        i.serving.append_codes(q, k, v, i.positions, i.slots, i.q_out, i.k, i.v, i.ks, i.vs, gq=i.gq, gk=i.gk)
        return {"q": i.q_out, "k": i.k, "v": i.v, "k_scale": i.ks, "v_scale": i.vs}
    rows = i.slots.shape[0]
    q, k, v = (t.float().reshape(rows, -1, d) for t in (q, k, v))
    if norm:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + eps) * i.gq.float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + eps) * i.gk.float()
    ang = i.positions.double()[:, None] * theta ** (-2.0 * torch.arange(d // 2, device=q.device).double() / d)
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    live = i.slots >= 0
    slots = i.slots[live].long()
    i.q_out.copy_(torch.where(live[:, None, None], _rotate(q, cos, sin).bfloat16(), i.q_out))
    _store(_rotate(k, cos, sin)[live], slots, i.k, i.ks)
    _store(v[live], slots, i.v, i.vs)
    return {"q": i.q_out, "k": i.k, "v": i.v, "k_scale": i.ks, "v_scale": i.vs}


def _attend(i, q, k, v, kv):
    """q [seqs, rows, nq, d] behind kv [seqs] cached tokens over k and v [seqs, keys, nkv, d], in 32 bits."""
    seqs, n, nq, d = q.shape
    keys, nkv = k.shape[1:3]
    q = q.float().view(seqs, n, nkv, nq // nkv, d).permute(0, 2, 3, 1, 4).reshape(seqs * nkv, -1, d)
    k, v = (t.permute(0, 2, 1, 3).reshape(seqs * nkv, keys, d) for t in (k, v))
    score = (torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)).view(seqs, nkv, nq // nkv, n, keys)
    late = torch.arange(keys, device=q.device) > kv[:, None, None] + torch.arange(n, device=q.device)[:, None]
    score.masked_fill_(late[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    out = torch.bmm(score.view(seqs * nkv, -1, keys), v).view(seqs, nkv, nq // nkv, n, d) / score.sum(-1, keepdim=True)
    return out.permute(0, 3, 1, 2, 4).reshape(seqs, n, nq, d).bfloat16()


def _values(codes, scale, pages):
    """The values of pages [seqs, pages], one token after the other."""
    x = codes[pages].float() * scale[pages].float()[:, :, None, :, None]
    return x.reshape(pages.shape[0], -1, *codes.shape[2:])


def _run_attention(i):
    if own:
        i.serving.attention_codes(i.q, i.out, i.q_indptr, i.kv_len, i.table, i.k, i.v, i.ks, i.vs)
        return i.out
    nq = i.q.shape[1]
    few = i.case["few"]
    together = [b for b, n in enumerate(i.new) if n == few]                # decoding sequences side by side, a few at a time
    most = max([1, max(1, (1 << 30) // (max(i.kv) + few) // (i.k.shape[2] * i.k.shape[3]))])
    for at in range(0, len(together), most):
        some = together[at:at + most]
        longest = _pages(max(i.kv[b] for b in some) + few)
        pages, kv = i.table[some, :longest].long(), i.kv_len[some].long()
        rows = i.q_indptr[some].long()[:, None] + torch.arange(few, device=kv.device)
        i.out[rows] = _attend(i, i.q[rows], _values(i.k, i.ks, pages), _values(i.v, i.vs, pages), kv)
    for b in (b for b, n in enumerate(i.new) if n != few):                 # prompts one by one, rows by memory
        total = i.kv[b] + i.new[b]
        pages = i.table[b:b + 1, :_pages(total)].long()
        k, v = _values(i.k, i.ks, pages)[:, :total], _values(i.v, i.vs, pages)[:, :total]
        step = max(1, (1 << 29) // (nq * total))
        for r in range(0, i.new[b], step):
            rows = slice(i.indptr[b] + r, min(i.indptr[b] + r + step, i.indptr[b + 1]))
            i.out[rows] = _attend(i, i.q[None, rows], k, v, i.kv_len[b:b + 1].long() + r)[0]
    return i.out


def _run_score(i):
    if own:
        i.serving.score(i.logits, i.tokens, i.logprob, entropy_out=i.entropy, top_ids=i.top_ids, top_logprobs=i.top_logprobs)
    else:
        rows, vocab = i.logits.shape
        x = i.logits.float() + 0.0
        bits = x.view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 20) + torch.arange(vocab - 1, -1, -1, device=x.device)
        ids = vocab - 1 - (order.topk(i.top_ids.shape[1], -1).values & ((1 << 20) - 1))      # larger first, then the lower id
        z = x.double()
        z -= z.amax(-1, keepdim=True)
        w = z.exp()
        total = w.sum(-1)
        i.entropy.copy_(total.log() - (w * z.clamp(min=-1e4)).sum(-1) / total)
        z -= total.log()[:, None]
        i.logprob.copy_(z.gather(1, i.tokens.long()[:, None])[:, 0])
        i.top_logprobs.copy_(z.gather(1, ids))
        i.top_ids.copy_(ids)
    return {"logprob": i.logprob, "entropy": i.entropy, "top_ids": i.top_ids, "top_logprobs": i.top_logprobs}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "append":
        nq, nkv, d, norm = HEADS[case["shape"]][:4]
        kv, new = _lengths(case)
        size, tokens = 4 if case["dtype"] == "fp32" else 2, sum(new)
        # rows in; queries, codes, scales of the pages out; slots and positions
        return {"bytes": tokens * d * (size * (nq + 2 * nkv) + 2 * nq + 2 * nkv) + 8 * (tokens + case["pad"]) +
                2 * nkv * sum(_touched(k, n) for k, n in zip(kv, new)), "flops": tokens * (nq + nkv) * d * (7 if norm else 3) + 4 * tokens * nkv * d}
    if case["op"] == "attention":
        nq, nkv, d = HEADS[case["shape"]][:3]
        kv, new = _lengths(case)
        pairs = sum(n * k + n * (n + 1) // 2 for k, n in zip(kv, new))
        keys, pages = sum(k + n for k, n in zip(kv, new)), sum(_pages(k + n) for k, n in zip(kv, new))
        return {"bytes": 4 * sum(new) * nq * d + 2 * keys * nkv * d + 2 * pages * nkv, "flops": 4 * pairs * nq * d}
    size = 4 if case["dtype"] == "fp32" else 2
    return {"bytes": case["rows"] * (case["vocab"] * size + 12 + 8 * case["top"]), "flops": 5 * case["rows"] * case["vocab"]}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    i = _inputs(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "score": _exact_score}[case["op"]](i)


def _to_code(x):
    """The nearest of the values that 4 significant bits and exponents from -6 hold; of two the one with the even last bit."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(i):
    nq, nkv, d, norm, theta, eps = HEADS[i.case["shape"]]
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
    q = i.q_out.double()
    q[live] = heads[:, :nq]
    out = {"q": q}
    slots = i.slots[live].tolist()
    begins = [0] + [r for r in range(1, len(slots)) if slots[r] != slots[r - 1] + 1 or slots[r] % PAGE == 0] + [len(slots)]
    for name, values, codes, scale in (("k", heads[:, nq:], i.k, i.ks), ("v", v, i.v, i.vs)):
        codes, scale = codes.double(), scale.double()
        for a, b in zip(begins, begins[1:]):                                # the rows of one page
            page, off = slots[a] // PAGE, slots[a] % PAGE
            most = values[a:b].abs().amax((0, 2))
            to = torch.exp2(torch.ceil(torch.log2(most / 448)).clamp(min=LOWEST))
            if off:
                to = torch.maximum(to, scale[page])
                codes[page, :off] = _to_code(codes[page, :off] * (scale[page] / to)[None, :, None])
            codes[page, off:off + b - a] = _to_code(values[a:b] / to[None, :, None])
            scale[page] = to
        out[name], out[name + "_scale"] = codes, scale
    return out


def _exact_attention(i):
    nq, nkv, d = HEADS[i.case["shape"]][:3]
    out = torch.zeros(i.indptr[-1], nq, d, dtype=torch.float64, device="cuda")
    for b, (kv, new) in enumerate(zip(i.kv, i.new)):
        slot = torch.arange(kv + new, device="cuda")
        page, at = i.table[b].long()[slot // PAGE], slot % PAGE
        for h in range(nkv):
            k, v = (c.view(torch.uint8)[page, at, h].view(torch.float8_e4m3fn).double() * s.view(torch.uint8)[page, h].view(torch.float8_e8m0fnu).double()[:, None]
                    for c, s in ((i.k, i.ks), (i.v, i.vs)))
            for g in range(h * (nq // nkv), (h + 1) * (nq // nkv)):
                for r in range(0, new, 2048):
                    q = i.q[i.indptr[b] + r:min(i.indptr[b] + r + 2048, i.indptr[b + 1]), g].double()
                    seen = slot[None, :] <= kv + r + torch.arange(q.shape[0], device="cuda")[:, None]
                    p = torch.where(seen, (q @ k.t()) * d ** -0.5, -math.inf).softmax(-1)
                    out[i.indptr[b] + r:i.indptr[b] + r + q.shape[0], g] = p @ v
    return out


def _exact_score(i):
    top = i.top_ids.shape[1]
    logprobs, entropies, ids, tops = [], [], [], []
    for r in range(0, i.logits.shape[0], 64):
        p = torch.log_softmax(i.logits[r:r + 64].double(), -1)
        logprobs.append(p.gather(1, i.tokens[r:r + 64, None].long())[:, 0])
        entropies.append(-torch.special.xlogy(p.exp(), p.exp()).sum(-1))
        best, at = i.logits[r:r + 64].float().sort(dim=-1, descending=True, stable=True)
        ids.append(at[:, :top].to(torch.int32))
        tops.append(p.gather(1, at[:, :top]))
    return {"logprob": torch.cat(logprobs), "entropy": torch.cat(entropies), "top_ids": torch.cat(ids), "top_logprobs": torch.cat(tops)}
