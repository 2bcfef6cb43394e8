"""Attention on the rollouts, as cases that can be timed and compared: over packed sequences with its gradient, for single
tokens on the paged KV pool with the prompt shared by a group's rollouts, and the eviction of cached tokens by the attention weight
that they have gathered.

  attend   queries of packed sequences over their keys, causal, grouped heads: prompts, survivors, chunks of a longer context
  grad     its gradient with respect to queries, keys and values (the survivors' training pass)
  decode   one token per rollout over its group's prompt pages and its own pages
  evict    the rollouts' caches cut to a budget of tokens, in place

Tensors are bf16 where the library's are (heads, KV pool) and fp32 elsewhere.  Lengths come from the case alone, values from the seed.
"""
import math

import torch

own = False

DEV = "cuda:0"


def listed():
    return [
        # the tiny configuration's prompts: a call of a few microseconds
        dict(name="attend_tiny", kind="attend", n=4, lo=16, hi=64, heads=4, kv=2, hd=64, context=0),
        # the prompts of a 1B-model batch, 64 of them, ragged
        dict(name="attend_prompts", kind="attend", n=64, lo=31, hi=512, heads=32, kv=8, hd=64, context=0),
        # chunks of prompts over what is cached of them already, 1.7B-model heads
        dict(name="attend_chunks", kind="attend", n=8, lo=1, hi=301, heads=16, kv=8, hd=128, context=3700),
        # a micro-batch of survivors of an 8B model, recomputed for the update
        dict(name="attend_survivors", kind="attend", n=4, lo=1024, hi=4096, heads=32, kv=8, hd=128, context=0),
        # the gradient at the tiny configuration's sizes
        dict(name="grad_tiny", kind="grad", n=4, lo=16, hi=64, heads=4, kv=2, hd=64, context=0),
        # the update on short survivors of a 1B model
        dict(name="grad_short", kind="grad", n=16, lo=65, hi=1000, heads=32, kv=8, hd=64, context=0),
        # the update on the survivors of an 8B model
        dict(name="grad_survivors", kind="grad", n=4, lo=1024, hi=4096, heads=32, kv=8, hd=128, context=0),
        # one prompt's rollouts, a few tokens in: latency
        dict(name="decode_one_prompt", kind="decode", groups=1, lo_g=8, hi_g=8, prefix_lo=200, prefix_hi=200, lo=1, hi=60, heads=32, kv=8, hd=64,
             page=16, weight=False),
        # a batch of a 1.7B model half way, pruned groups of different sizes, weights gathered
        dict(name="decode_batch", kind="decode", groups=64, lo_g=4, hi_g=8, prefix_lo=100, prefix_hi=600, lo=1, hi=2000, heads=16, kv=8, hd=128,
             page=16, weight=True),
        # long prompts shared by 16 rollouts each, 8B-model heads
        dict(name="decode_long_prompts", kind="decode", groups=4, lo_g=16, hi_g=16, prefix_lo=9000, prefix_hi=16384, lo=100, hi=1000, heads=32, kv=8,
             hd=128, page=16, weight=True),
        # the tiny configuration's caches, halved
        dict(name="evict_tiny", kind="evict", rows=32, lo=20, hi=64, budget=32, first=2, recent=8, layers=2, kv=2, hd=64, page=16),
        # a 1B-model batch's caches (all layers) cut to half the checkpoint length
        dict(name="evict_batch", kind="evict", rows=128, lo=100, hi=1024, budget=256, first=4, recent=64, layers=16, kv=8, hd=64, page=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "grad", "decode", "evict"])
    kv, hd = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    if kind in ("attend", "grad"):
        n, hi = _log_int(rng, 1, 64), _log_int(rng, 16, 4096)
        heads = kv * rng.choice([1, 2, 3, 4])
        hi = max(8, min(hi, int(math.sqrt(4 * 4096 * 4096 * 32 / (n * heads)))))
        context = _log_int(rng, 1, 2048) if kind == "attend" and rng.random() < 0.3 and hi * n < 8192 else 0
        return dict(kind=kind, n=n, lo=_log_int(rng, 1, hi), hi=hi, heads=heads, kv=kv, hd=hd, context=context)
    if kind == "decode":
        heads, groups = kv * rng.choice([1, 2, 3, 4, 8]), _log_int(rng, 1, 32)
        hi_g, prefix, hi = rng.randint(1, 16), _log_int(rng, 1, 4096), _log_int(rng, 1, 2048)
        return dict(kind=kind, groups=groups, lo_g=rng.randint(1, hi_g), hi_g=hi_g, prefix_lo=_log_int(rng, 1, prefix), prefix_hi=prefix,
                    lo=_log_int(rng, 1, hi), hi=hi, heads=heads, kv=kv, hd=hd, page=rng.choice([8, 16, 32]), weight=rng.random() < 0.5)
    hi, rows = _log_int(rng, 40, 4096), _log_int(rng, 1, 96)
    budget = max(32, int(hi * rng.uniform(0.2, 0.8)))
    return dict(kind=kind, rows=min(rows, 96 * 1024 // hi + 1), lo=_log_int(rng, 1, hi), hi=hi, budget=budget, first=rng.randint(0, 4),
                recent=rng.randint(0, budget // 2), layers=rng.randint(1, 16), kv=kv, hd=hd, page=rng.choice([8, 16, 32]))


def _lengths(n, lo, hi):
    """n lengths spread over [lo, hi], the longest among them."""
    return [hi - int((hi - lo + 1) * ((0.6180339887498949 * i) % 1.0)) for i in range(n)]


def _offsets(lengths):
    at = [0]
    for x in lengths:
        at.append(at[-1] + x)
    return torch.tensor(at, dtype=torch.int64, device=DEV)


def _packed_lengths(case):
    """Queries and keys of every sequence: with a context, the keys of up to so many earlier tokens come before the queries'."""
    nq = _lengths(case["n"], case["lo"], case["hi"])
    before = _lengths(case["n"], case["context"] // 8, case["context"]) if case["context"] else [0] * case["n"]
    return nq, [a + b for a, b in zip(nq, before)]


def _prepare_packed(case, g):
    nq, nk = _packed_lengths(case)
    H, KV, hd = case["heads"], case["kv"], case["hd"]
    if case["context"]:
        q = torch.randn(sum(nq), H, hd, generator=g, device=DEV).to(torch.bfloat16)
        kv = torch.randn(sum(nk), 2 * KV, hd, generator=g, device=DEV).to(torch.bfloat16)
        k, v = kv[:, :KV], kv[:, KV:]
    else:       # slices of one projection's output, as a model hands them on
        qkv = torch.randn(sum(nq), H + 2 * KV, hd, generator=g, device=DEV).to(torch.bfloat16)
        q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    state = dict(kind=case["kind"], q=q, k=k, v=v, cu_q=_offsets(nq), cu_k=_offsets(nk) if case["context"] else None, longest_q=max(nq), longest_k=max(nk))
    if case["kind"] == "grad":
        state["out"], state["lse"] = _attend(state)
        state["grad_out"] = torch.randn(q.shape, generator=g, device=DEV).to(torch.bfloat16)
    return state


def _decode_lengths(case):
    sizes = _lengths(case["groups"], case["lo_g"], case["hi_g"])
    return sizes, _lengths(case["groups"], case["prefix_lo"], case["prefix_hi"]), _lengths(sum(sizes), case["lo"], case["hi"])


def _tables(case, lengths, pages, first):
    """Block tables: rows of the pages from `first` on in the order of `pages`, -1 past a row's length."""
    per, width = case["page"], -(-max(lengths) // case["page"])
    n = torch.tensor([-(-x // per) for x in lengths], device=DEV)
    at = first + torch.cumsum(n, 0)[:, None] - n[:, None] + torch.arange(width, device=DEV)
    inside = torch.arange(width, device=DEV) < n[:, None]
    return torch.where(inside, pages[at.clamp(max=pages.numel() - 1)], -1).to(torch.int32), int(n.sum())


def _prepare_decode(case, g):
    sizes, prefix, lengths = _decode_lengths(case)
    total = sum(-(-x // case["page"]) for x in prefix + lengths)
    pages = torch.randperm(total, generator=g, device=DEV)
    prefix_table, used = _tables(case, prefix, pages, 0)
    table, _ = _tables(case, lengths, pages, used)
    kv = torch.randn(2, 2, total, case["page"], case["kv"], case["hd"], generator=g, device=DEV).to(torch.bfloat16)
    q = torch.randn(len(lengths), case["heads"], case["hd"], generator=g, device=DEV).to(torch.bfloat16)
    state = dict(kind="decode", q=q, kv=kv, layer=1, table=table, seq_len=torch.tensor(lengths, dtype=torch.int32, device=DEV), prefix_table=prefix_table,
                 prefix_len=torch.tensor(prefix, dtype=torch.int32, device=DEV), group_offsets=_offsets(sizes), weight=case["weight"])
    if case["weight"]:      # what earlier tokens have gathered
        state["gathered"] = torch.rand(table.shape[0], table.shape[1] * case["page"], generator=g, device=DEV)
        state["prefix_gathered"] = torch.rand(prefix_table.shape[0], prefix_table.shape[1] * case["page"], generator=g, device=DEV)
    return state


def _prepare_evict(case, g):
    lengths = _lengths(case["rows"], case["lo"], case["hi"])
    total = sum(-(-x // case["page"]) for x in lengths)
    table, _ = _tables(case, lengths, torch.randperm(total, generator=g, device=DEV), 0)
    kv = torch.randn(case["layers"], 2, total, case["page"], case["kv"], case["hd"], generator=g, device=DEV, dtype=torch.bfloat16)
    # few tokens hold most of the weight, and some hold none at all: equal weights
    weight = torch.rand(table.shape[0], table.shape[1] * case["page"], generator=g, device=DEV) ** 8
    weight = torch.where(weight < 1e-4, torch.zeros_like(weight), weight)
    return dict(kind="evict", kv=kv, table=table, seq_len=torch.tensor(lengths, dtype=torch.int32, device=DEV), weight=weight, budget=case["budget"],
                first=case["first"], recent=case["recent"])


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return {"attend": _prepare_packed, "grad": _prepare_packed, "decode": _prepare_decode, "evict": _prepare_evict}[case["kind"]](case, g)


def _padded(x, cu, longest):
    """Packed rows [T, heads, hd] as fp32 [sequences, heads, longest, hd]."""
    rows = (cu[:-1, None] + torch.arange(longest, device=x.device)).clamp(max=x.shape[0] - 1)
    return x[rows].float().transpose(1, 2).contiguous()


def _tokens(cu, T):
    """Sequence and position of every packed row."""
    t = torch.arange(T, device=cu.device)
    seq = torch.searchsorted(cu, t, right=True) - 1
    return seq, t - cu[seq]


def _scores(s):
    """Scaled products of every query with every key [sequences, kv heads, heads of one, queries, keys], -inf where it may not look, and
    the operands in 32 bits."""
    cu_q, cu_k = s["cu_q"], s["cu_q"] if s["cu_k"] is None else s["cu_k"]
    q, k, v = _padded(s["q"], cu_q, s["longest_q"]), _padded(s["k"], cu_k, s["longest_k"]), _padded(s["v"], cu_k, s["longest_k"])
    n, H, L, hd = q.shape
    q = q.view(n, k.shape[1], -1, hd)
    z = (torch.matmul(q, k.transpose(2, 3).contiguous()) * hd ** -0.5).view(n, k.shape[1], -1, L, k.shape[2])
    nq, nk = (cu_q[1:] - cu_q[:-1])[:, None, None], (cu_k[1:] - cu_k[:-1])[:, None, None]
    i, j = torch.arange(L, device=z.device)[:, None], torch.arange(z.shape[4], device=z.device)
    sees = (j < nk) & (i < nq) & (j + nq <= i + nk)
    return z.masked_fill(~sees[:, None, None], -math.inf), q, k, v


def _attend(s):
    z, q, k, v = _scores(s)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(q.shape[:3] + (-1,)), v).view(p.shape[:4] + (-1,)) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + torch.log(total))[..., 0]
    seq, at = _tokens(s["cu_q"], s["q"].shape[0])
    return o.flatten(1, 2)[seq, :, at].to(torch.bfloat16), lse.flatten(1, 2)[seq, :, at].t().contiguous()


def _grad(s):
    z, q, k, v = _scores(s)
    do = _padded(s["grad_out"], s["cu_q"], s["longest_q"]).view(q.shape)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous()).view(p.shape)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["q"].shape[2] ** -0.5
    p, ds = p.view(q.shape[:3] + (-1,)), ds.view(q.shape[:3] + (-1,))
    dv, dk, dq = torch.matmul(p.transpose(2, 3).contiguous(), do), torch.matmul(ds.transpose(2, 3).contiguous(), q), torch.matmul(ds, k)
    seq, at = _tokens(s["cu_q"], s["q"].shape[0])
    dq = dq.view(dq.shape[0], -1, s["longest_q"], dq.shape[3])
    return tuple(x[seq, :, at].to(torch.bfloat16) for x in (dq, dk, dv))


def _cached(kv, layer, table):
    """Cached keys and values of every row of a block table, fp32 [rows, kv heads, tokens, hd]."""
    x = kv[layer][:, table.clamp(min=0).long()].float()
    return x.flatten(2, 3).transpose(2, 3).contiguous()


def _decode(s):
    q, kv = s["q"], s["kv"]
    N, H, hd = q.shape
    group = torch.searchsorted(s["group_offsets"], torch.arange(N, device=q.device), right=True) - 1
    pk, pv = _cached(kv, s["layer"], s["prefix_table"])
    k, v = _cached(kv, s["layer"], s["table"])
    keys, values = torch.cat([pk[group], k], 2), torch.cat([pv[group], v], 2)
    P, C = pk.shape[2], k.shape[2]
    qs = q.float().view(N, k.shape[1], -1, hd)
    z = torch.matmul(qs, keys.transpose(2, 3).contiguous()) * hd ** -0.5
    sees = torch.cat([torch.arange(P, device=q.device) < s["prefix_len"][group][:, None], torch.arange(C, device=q.device) < s["seq_len"][:, None]], 1)
    z = z.masked_fill(~sees[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    out, lse = torch.matmul(p, values) / total, (top + torch.log(total)).reshape(N, H)
    out = out.reshape(N, H, hd).to(torch.bfloat16)
    if not s["weight"]:
        return out, lse
    w = (p / total).sum((1, 2))
    members = (group == torch.arange(pk.shape[0], device=q.device)[:, None]).float()
    inside, prefix_inside = torch.arange(C, device=q.device) < s["seq_len"][:, None], torch.arange(P, device=q.device) < s["prefix_len"][:, None]
    own_w = torch.where(inside, s["gathered"] + w[:, P:], torch.zeros_like(w[:, P:]))
    prefix_w = torch.where(prefix_inside, s["prefix_gathered"] + torch.matmul(members, w[:, :P]), torch.zeros_like(s["prefix_gathered"]))
    return out, lse, own_w, prefix_w


def _evict(s):
    kv, table, length, weight = s["kv"], s["table"], s["seq_len"].long()[:, None], s["weight"]
    page, C = kv.shape[3], weight.shape[1]
    t = torch.arange(C, device=kv.device)
    left = length.clamp(max=s["budget"])
    fixed = (t < s["first"]) | (t >= length - s["recent"])
    rank = torch.where(fixed, torch.full_like(weight, math.inf), weight)
    rank = torch.where(t < length, rank, torch.full_like(weight, -math.inf))
    order = torch.sort(rank, dim=1, descending=True, stable=True)[1]
    kept = torch.zeros_like(weight, dtype=torch.bool).scatter_(1, order, t < left)
    # the k-th kept token behind the cut goes to the k-th slot before it that has come free
    moves, hole = kept & (t >= left), ~kept & (t < left)
    source = torch.sort((~moves).to(torch.uint8), dim=1, stable=True)[1]
    k = torch.cumsum(hole.long(), 1) - 1
    position = torch.where(hole, torch.gather(source, 1, k.clamp(min=0)), t.expand_as(kept))
    after = t < left
    slot = table.clamp(min=0).long().repeat_interleave(page, 1) * page + t % page
    flat = kv.flatten(2, 3)
    source = torch.gather(slot, 1, torch.where(after, position, position[:, :1]))
    flat[:, :, torch.where(after, slot, slot[:, :1])] = flat[:, :, source]      # past a row's end: its first slot once more
    pages = torch.arange(table.shape[1], device=kv.device) * page < left
    return (kv, torch.where(pages, table, -1), left[:, 0].to(torch.int32), torch.where(after, torch.gather(weight, 1, position), torch.zeros_like(weight)),
            torch.where(after, position, -1).to(torch.int32))


def _run_own(s):
    import paper_2603_24840_amd as A

    if s["kind"] == "attend":
        return A.arrol_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"])
    if s["kind"] == "grad":
        grad = A.arrol_attention_grad(s["q"], s["k"], s["v"], s["out"], s["lse"], s["grad_out"], s["cu_q"], s["cu_k"])
        return grad["grad_q"], grad["grad_k"], grad["grad_v"]
    if s["kind"] == "decode":
        got = A.arrol_decode_attention(s["q"], s["kv"], s["layer"], s["table"], s["seq_len"], s["prefix_table"], s["prefix_len"], s["group_offsets"],
                                       want_weight=s["weight"], weight=s.get("gathered"), prefix_weight=s.get("prefix_gathered"))
        return (got["out"], got["lse"]) + ((got["weight"], got["prefix_weight"]) if s["weight"] else ())
    got = A.arrol_evict(s["kv"], s["table"], s["seq_len"], s["weight"], s["budget"], n_first=s["first"], n_recent=s["recent"])
    return s["kv"], got["block_table"], got["seq_len"], got["weight"], got["position"]


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _attend, "grad": _grad, "decode": _decode, "evict": _evict}[state["kind"]](state)


def work(case):
    hd, KV = case["hd"], case["kv"]
    if case["kind"] in ("attend", "grad"):
        H = case["heads"]
        nq, nk = _packed_lengths(case)
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(nq, nk))
        if case["kind"] == "attend":
            return {"bytes": 2 * hd * (2 * H * sum(nq) + 2 * KV * sum(nk)) + 4 * H * sum(nq), "flops": 4 * hd * H * pairs}
        return {"bytes": 2 * hd * (4 * H * sum(nq) + 4 * KV * sum(nk)) + 4 * H * sum(nq), "flops": 10 * hd * H * pairs}
    if case["kind"] == "decode":
        sizes, prefix, lengths = _decode_lengths(case)
        tokens, N = sum(prefix) + sum(lengths), len(lengths)
        looked = sum(lengths) + sum(a * b for a, b in zip(sizes, prefix))
        return {"bytes": 4 * KV * hd * tokens + N * case["heads"] * (4 * hd + 4) + (8 * tokens if case["weight"] else 0), "flops": 4 * hd * case["heads"] * looked}
    # of the tokens that stay, those behind the cut are moved: the recent ones, and the heavy ones' share
    moved = 0
    for n in _lengths(case["rows"], case["lo"], case["hi"]):
        if n > case["budget"]:
            recent, heavy = min(case["recent"], n - case["budget"]), case["budget"] - case["first"] - case["recent"]
            moved += recent + heavy * max(0, n - case["recent"] - case["budget"]) / max(1, n - case["first"] - case["recent"])
    tokens = sum(_lengths(case["rows"], case["lo"], case["hi"]))
    return {"bytes": int(moved * case["layers"] * 2 * KV * hd * 2 * 2 + 4 * tokens), "flops": 0}


def _exact_packed(s, grad):
    """Sequence by sequence and head by head in 64 bits; the gradient by differentiating that."""
    cu_q = s["cu_q"].tolist()
    cu_k = cu_q if s["cu_k"] is None else s["cu_k"].tolist()
    q, k, v = (x.double() for x in (s["q"], s["k"], s["v"]))
    H, KV, hd = q.shape[1], k.shape[1], q.shape[2]
    out, lse = torch.zeros_like(q), torch.full((H, q.shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    grads = [torch.zeros_like(x) for x in (q, k, v)]
    for a, b, c, d in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
        bias = torch.zeros(b - a, d - c, dtype=torch.float64, device=DEV)
        bias.masked_fill_(torch.ones_like(bias, dtype=torch.bool).triu((d - c) - (b - a) + 1), -math.inf)
        for h in range(H):
            x, y, w = (t.clone().requires_grad_(grad) for t in (q[a:b, h], k[c:d, h * KV // H], v[c:d, h * KV // H]))
            z = torch.mm(x, y.t()) / math.sqrt(hd) + bias
            o = torch.mm(torch.softmax(z, 1), w)
            if not grad:
                out[a:b, h], lse[h, a:b] = o, torch.logsumexp(z, 1)
                continue
            for total, part, rows, head in zip(grads, torch.autograd.grad(o, (x, y, w), s["grad_out"][a:b, h].double()), ((a, b), (c, d), (c, d)),
                                               (h, h * KV // H, h * KV // H)):
                total[rows[0]:rows[1], head] += part
    return tuple(grads) if grad else (out, lse)


def _exact_decode(s):
    q, kv, page = s["q"].double(), s["kv"][s["layer"]], s["kv"].shape[3]
    N, H, hd = q.shape
    per = H // kv.shape[3]
    out, lse = torch.zeros_like(q), torch.zeros(N, H, dtype=torch.float64, device=DEV)
    weight, prefix_weight = ((s[x].double().clone() for x in ("gathered", "prefix_gathered")) if s["weight"] else (None, None))
    offsets, prefix, lengths = s["group_offsets"].tolist(), s["prefix_len"].tolist(), s["seq_len"].tolist()
    for g in range(len(prefix)):
        shared = kv[:, s["prefix_table"][g, :-(-prefix[g] // page)].long()].flatten(1, 2)[:, :prefix[g]].double()
        if s["weight"]:
            prefix_weight[g, prefix[g]:] = 0
        for r in range(offsets[g], offsets[g + 1]):
            mine = kv[:, s["table"][r, :-(-lengths[r] // page)].long()].flatten(1, 2)[:, :lengths[r]].double()
            k, v = torch.cat([shared, mine], 1).transpose(1, 2).repeat_interleave(per, 1)
            z = (k * q[r][:, None]).sum(-1) / math.sqrt(hd)
            p = torch.softmax(z, -1)
            out[r], lse[r] = (p[..., None] * v).sum(1), torch.logsumexp(z, -1)
            if s["weight"]:
                p = p.sum(0)
                prefix_weight[g, :prefix[g]] += p[:prefix[g]]
                weight[r, :lengths[r]] += p[prefix[g]:]
                weight[r, lengths[r]:] = 0
    return (out, lse, weight, prefix_weight) if s["weight"] else (out, lse)


def _exact_evict(s):
    """Row by row; the pool is moved, not computed."""
    lengths, weights, page = s["seq_len"].tolist(), s["weight"].tolist(), s["kv"].shape[3]
    table = s["table"].clone()
    weight, position = torch.zeros_like(s["weight"], dtype=torch.float64), torch.full(s["weight"].shape, -1, dtype=torch.int32)
    for r, n in enumerate(lengths):
        left = min(n, s["budget"])
        table[r, -(-left // page):] = -1
        slots = list(range(left))
        if n > left:
            between = range(s["first"], n - s["recent"])
            heavy = sorted(between, key=lambda t: (-weights[r][t], t))[:left - s["first"] - s["recent"]]
            stay = set(heavy) | set(range(s["first"])) | set(range(n - s["recent"], n))
            behind = iter(sorted(t for t in stay if t >= left))
            slots = [t if t in stay else next(behind) for t in range(left)]
        weight[r, :left] = torch.tensor([weights[r][t] for t in slots], dtype=torch.float64, device=weight.device)
        position[r, :left] = torch.tensor(slots, dtype=torch.int32)
    return None, table, s["seq_len"].clamp(max=s["budget"]), weight, position.to(DEV)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "decode":
        return _exact_decode(s)
    if case["kind"] == "evict":
        return _exact_evict(s)
    return _exact_packed(s, case["kind"] == "grad")
